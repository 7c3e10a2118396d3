// Eviction: of each request, layer and KV head the most recent tokens stay, and of the others those of
// largest weight, ties by position. Their rows and weights move, in order, to the front of `to`.
//
// Two launches. The first finds what stays: a workgroup for each (layer, request, head) finds the
// weight from which on tokens stay by three passes over the weights' bits, 11, 11 and 10 at a time, counting
// them in LDS; then each wave goes through a sixteenth of the tokens, in order, once to count those that stay and once
// to write their positions. The second moves rows and weights, bound by memory: what stays is read
// and written once.
//
// `to` may name the pages that the rows are on already. A row never moves back, so a workgroup that takes
// the rows of a unit in order, and has read a chunk whole before it writes it, overwrites nothing that is still to be
// read; a unit's planes, 128 bytes of each row, and the weights are workgroups of their own. Where a
// request's pages are all others there is no order to keep: a unit's workgroups then take 64 tokens at a time,
// all of their rows, whose places 64 lanes find for all.
//
// Measured, to other pages: 16 requests of 250 to 8,000 tokens to a quarter, 2 layers of 8 heads, 16 us for the first
// (with 512 threads 18) and 59 for the second (275 MB, 4.7 TB/s), 78 a call; one of 2,049 to half, 8 layers, 10 and 15
// (chains of trips to memory; bytes take 12), 27 to 29 a call. In place 139 and 96 a call: one workgroup a unit and 128
// bytes of its rows, in order. Replayed from a graph a call takes 2 to 4 us more than its kernels; so timed, moving by 512
// threads instead of 256, or with 16 rows of a lane under way, made the one request's call 38 to 51 us, where an earlier
// selection and these movers took 33.
#include <hip/hip_runtime.h>

#include "lds_fetch.hpp"
#include "weights.hpp"

namespace ptsd {
namespace {

typedef unsigned int v4u __attribute__((ext_vector_type(4)));

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 2048;
constexpr int kReads = 4;        // weights of a lane under way
constexpr int kCached = 12288;  // weights that stay in LDS between passes; of longer requests they are read again
constexpr int kMoveThreads = 256;
constexpr int kSlice = 8;       // 16-byte pieces of a row that a workgroup moves
constexpr int kDeep = 8;        // rows of a lane under way
constexpr int kTokens = 64;     // that a workgroup moves at once where there is no order to keep
constexpr int kMovers = 16;     // workgroups of a compute unit
constexpr int kMostParts = 16;

// What a request keeps: n tokens, m of them, the last `recent` for sure.
struct Kept {
    int32_t n, m, recent;
};
__device__ inline Kept kept_of(const KeepPlan& p, int r) {
    const int64_t limit = (int64_t)p.max_blocks * p.div.page;
    const int32_t context = p.context[r], keep = p.keep[r];
    Kept k;
    k.n = context < 0 ? 0 : context < limit ? context : (int32_t)limit;
    k.m = keep < p.max_keep ? keep : p.max_keep;
    k.m = k.m < 0 ? 0 : k.m < k.n ? k.m : k.n;
    k.recent = p.recent < k.m ? p.recent : k.m;
    return k;
}

// A position's block and slot in a table's row, or false.
__device__ inline bool locate(const KeepPlan& p, const int32_t* table, int32_t i, int32_t& block, uint32_t& slot) {
    const uint32_t column = div_page((uint32_t)i, p.div);
    block = table[column];
    slot = (uint32_t)i - column * p.div.page;
    return block >= 0 && block < p.blocks;
}

__device__ inline float* weight_at(const KeepPlan& p, int layer, int head, int32_t block, uint32_t slot) {
    return p.weights + (((int64_t)layer * p.blocks + block) * p.heads + head) * p.div.page + slot;
}

// A weight's place in the order, as a whole number: NaN last, both zeros alike.
__device__ inline uint32_t order_of(float x) {
    if (x != x) return ~0u;
    const uint32_t bits = __float_as_uint(x + 0.f);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

// Sums of all threads' values before a thread's, in thread order.
__device__ inline uint32_t scan(uint32_t x, uint32_t* s_wave) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t sum = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(sum, d);
        if (lane >= d) sum += o;
    }
    __syncthreads();  // s_wave is free
    if (lane == 63) s_wave[wave] = sum;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int i = 0; i < kSelectWaves; ++i)
        if (i < wave) before += s_wave[i];
    return before + sum - x;
}

__global__ __launch_bounds__(kSelectThreads) void k_keep_select(KeepPlan p) {
    __shared__ uint32_t s_order[kCached];
    __shared__ uint32_t s_count[kBins];
    __shared__ uint32_t s_wave[kSelectWaves];
    __shared__ uint32_t s_sure[kSelectWaves], s_ties[kSelectWaves];
    __shared__ uint32_t s_bin, s_above;
    const int tid = threadIdx.x;
    const int unit = blockIdx.x, head = unit % p.heads, r = unit / p.heads % p.R, layer = unit / p.heads / p.R;
    const Kept k = kept_of(p, r);
    if (layer == 0 && head == 0 && tid == 0) p.context_out[r] = k.m;
    if (k.m == 0) return;
    const int32_t* const table = p.from + (int64_t)r * p.max_blocks;
    int32_t* const source = p.source + (int64_t)unit * p.max_keep;
    const int32_t rest = k.n - k.recent;                   // candidates
    uint32_t want = (uint32_t)(k.m - k.recent);            // of them
    // weights i0 + tid, .. + 1,024, ..: several at once, their pages first
    auto read = [&](int32_t i0, uint32_t (&x)[kReads]) {
        int32_t block[kReads];
        uint32_t slot[kReads];
        bool there[kReads];
#pragma unroll
        for (int u = 0; u < kReads; ++u) {
            const int32_t i = i0 + u * kSelectThreads + tid;
            there[u] = locate(p, table, i < k.n ? i : k.n - 1, block[u], slot[u]);
        }
        float w[kReads];
#pragma unroll
        for (int u = 0; u < kReads; ++u)
            w[u] = *weight_at(p, layer, head, there[u] ? block[u] : 0, there[u] ? slot[u] : 0);
#pragma unroll
        for (int u = 0; u < kReads; ++u) x[u] = there[u] ? order_of(w[u]) : 0u;
    };
    const bool cached = rest <= kCached, all_stay = (int32_t)want == rest, none = want == 0;
    uint32_t border = 0;  // tokens above it stay, and of those at it the first `want`
    if (!all_stay && !none) {
        for (int pass = 0; pass < 3; ++pass) {
            const int bits = pass < 2 ? 11 : 10, low = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            for (int b = tid; b < kBins; b += kSelectThreads) s_count[b] = 0;
            __syncthreads();
            for (int32_t i0 = 0; i0 < rest; i0 += kSelectThreads * kReads) {
                uint32_t x[kReads];
                if (pass == 0 || !cached) {
                    read(i0, x);
                } else {
#pragma unroll
                    for (int u = 0; u < kReads; ++u) {
                        const int32_t i = i0 + u * kSelectThreads + tid;
                        x[u] = s_order[i < rest ? i : 0];
                    }
                }
#pragma unroll
                for (int u = 0; u < kReads; ++u) {
                    const int32_t i = i0 + u * kSelectThreads + tid;
                    if (i >= rest) break;
                    if (pass == 0 && cached) s_order[i] = x[u];
                    if (pass == 0 || x[u] >> (low + bits) == border >> (low + bits))
                        atomicAdd(&s_count[(x[u] >> low) & ((1u << bits) - 1)], 1u);
                }
            }
            __syncthreads();
            // thread t has the bins 2047 - 2 t and 2046 - 2 t: the largest first
            constexpr int kOf = kBins / kSelectThreads;
            uint32_t mine[kOf], sum = 0;
#pragma unroll
            for (int j = 0; j < kOf; ++j) {
                mine[j] = s_count[kBins - 1 - (tid * kOf + j)];
                sum += mine[j];
            }
            uint32_t above = scan(sum, s_wave);
#pragma unroll
            for (int j = 0; j < kOf; ++j) {
                if (above < want && above + mine[j] >= want) {
                    s_bin = kBins - 1 - (tid * kOf + j);
                    s_above = above;
                }
                above += mine[j];
            }
            __syncthreads();
            border |= s_bin << low;
            want -= s_above;
            __syncthreads();
        }
    }
    // In order, a wave a sixteenth of the tokens, 64 at a time: how many are above the border, and at it; then, with
    // the sums of the waves before, the positions that stay.
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int32_t each = ((k.n + 63) / 64 + kSelectWaves - 1) / kSelectWaves * 64;
    const int32_t from = wave * each, until = from + each < k.n ? from + each : k.n;
    auto order = [&](int32_t i) {
        if (cached) return s_order[i];
        int32_t block;
        uint32_t slot;
        return locate(p, table, i, block, slot) ? order_of(*weight_at(p, layer, head, block, slot)) : 0u;
    };
    const bool choose = !all_stay && !none;
    uint32_t sure = 0, ties = 0;
    for (int32_t i0 = from; i0 < until; i0 += 64) {
        const int32_t i = i0 + lane;
        const uint32_t x = choose && i < rest ? order(i) : 0u;
        const bool stays = i < k.n && (i >= rest || all_stay || (choose && x > border));
        sure += __popcll(__ballot(stays));
        ties += __popcll(__ballot(choose && i < rest && x == border));
    }
    if (lane == 0) {
        s_sure[wave] = sure;
        s_ties[wave] = ties;
    }
    __syncthreads();
    uint32_t done = 0, tied = 0;  // of the waves before: those that stay, and at the border
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
        if (w >= wave) break;
        const uint32_t left = want > tied ? want - tied : 0u;
        done += s_sure[w] + (s_ties[w] < left ? s_ties[w] : left);
        tied += s_ties[w];
    }
    const uint64_t below = (1ull << lane) - 1;
    for (int32_t i0 = from; i0 < until; i0 += 64) {
        const int32_t i = i0 + lane;
        const uint32_t x = choose && i < rest ? order(i) : 0u;
        const bool tie = choose && i < rest && x == border;
        const uint64_t at_border = __ballot(tie);
        const bool stays = i < k.n && (i >= rest || all_stay || (choose && x > border) ||
                                       (tie && tied + __popcll(at_border & below) < want));
        tied += __popcll(at_border);
        const uint64_t staying = __ballot(stays);
        if (stays) source[done + __popcll(staying & below)] = i;
        done += __popcll(staying);
    }
}

// Whether a request's first m tokens go to pages other than those of the same columns.
__device__ inline bool apart(const KeepPlan& p, int r, int32_t m) {
    const int32_t* const from = p.from + (int64_t)r * p.max_blocks;
    const int32_t* const to = p.to + (int64_t)r * p.max_blocks;
    bool same = false;
    const int32_t columns = (int32_t)div_page((uint32_t)(m - 1), p.div) + 1;
    for (int32_t c = threadIdx.x; c < columns; c += kMoveThreads) same |= from[c] == to[c];
    return !__syncthreads_or(same);
}

// kPower: bytes of a row's exponents. Workgroups of a unit: its planes' slices, then the weights, `parts` of each.
template <int kPower>
__global__ __launch_bounds__(kMoveThreads) void k_keep_move(KeepPlan p, int planes, int slices, int columns, int parts,
                                                            PageDiv pieces) {
    const int part = blockIdx.x % parts, kinds = planes * slices + 1, kind = blockIdx.x / parts % kinds;
    const int unit = blockIdx.x / parts / kinds;
    const int head = unit % p.heads, r = unit / p.heads % p.R, layer = unit / p.heads / p.R;
    const Kept k = kept_of(p, r);
    if (k.m == 0) return;
    const int32_t* const from = p.from + (int64_t)r * p.max_blocks;
    const int32_t* const to = p.to + (int64_t)r * p.max_blocks;
    const int32_t* const source = p.source + (int64_t)unit * p.max_keep;
    if (apart(p, r, k.m)) {
        __shared__ uint32_t s_from[2][kTokens], s_to[2][kTokens];  // rows of a plane, counted from its first
        constexpr uint32_t kNone = ~0u;
        const int workers = kinds * parts, me = kind * parts + part;
        auto find = [&](int32_t i0, int buffer) {
            if (threadIdx.x >= kTokens) return;
            const int32_t i = i0 + threadIdx.x;
            int32_t block, to_block;
            uint32_t slot, to_slot;
            const bool there = i < k.m && locate(p, from, source[i], block, slot) && locate(p, to, i, to_block, to_slot);
            s_from[buffer][threadIdx.x] = there ? ((uint32_t)block * p.heads + head) * p.div.page + slot : kNone;
            s_to[buffer][threadIdx.x] = there ? ((uint32_t)to_block * p.heads + head) * p.div.page + to_slot : 0u;
        };
        // a row's place: slabs are not always a whole number of rows (4 bits)
        auto row_at = [&](uint32_t row) {
            if (!kPower) return (int64_t)row * p.row;
            const uint32_t block = div_page(row, p.slab_rows);
            return (int64_t)block * p.slab + (int64_t)(row - block * p.slab_rows.page) * p.row;
        };
        uint8_t* const k0 = p.k + (int64_t)layer * p.layer;
        uint8_t* const v0 = planes > 1 ? p.v + (int64_t)layer * p.layer : nullptr;
        float* const weights = p.weights + (int64_t)layer * p.blocks * p.heads * p.div.page;
        const uint32_t all = kTokens * pieces.page;  // 16-byte pieces of 64 tokens
        int buffer = 0;
        find(me * kTokens, 0);
        for (int32_t i0 = me * kTokens; i0 < k.m; i0 += workers * kTokens, buffer ^= 1) {
            __syncthreads();
            for (uint32_t first = threadIdx.x; first < all; first += kMoveThreads * kDeep) {
                v4u x[kDeep];
                uint8_t* at[kDeep];
#pragma unroll
                for (int u = 0; u < kDeep; ++u) {
                    const uint32_t piece = first + u * kMoveThreads;
                    at[u] = nullptr;
                    if (piece >= all) continue;
                    const uint32_t token = div_page(piece, pieces), c = piece - token * pieces.page;
                    const uint32_t row = s_from[buffer][token];
                    if (row == kNone) continue;
                    uint8_t* const base = c < (uint32_t)columns ? k0 + c * 16 : v0 + (c - columns) * 16;
                    x[u] = __builtin_nontemporal_load((const v4u*)(base + row_at(row)));
                    at[u] = base + row_at(s_to[buffer][token]);
                }
                if (first == threadIdx.x) find(i0 + workers * kTokens, buffer ^ 1);  // the next tokens' rows
#pragma unroll
                for (int u = 0; u < kDeep; ++u)
                    if (at[u]) __builtin_nontemporal_store(x[u], (v4u*)at[u]);
            }
            const int token = threadIdx.x % kTokens, what = threadIdx.x / kTokens;
            const uint32_t row = s_from[buffer][token], to_row = s_to[buffer][token];
            if (row == kNone) continue;
            if (what == 0) weights[to_row] = weights[row];
            if (kPower && (what == 1 || what == 2)) {
                uint8_t* const base = (what == 1 ? k0 : v0) + p.powers;
                const uint32_t a = div_page(row, p.slab_rows), b = div_page(to_row, p.slab_rows);
                const uint8_t* const x = base + (int64_t)a * p.slab + (row - a * p.slab_rows.page) * kPower;
                uint8_t* const y = base + (int64_t)b * p.slab + (to_row - b * p.slab_rows.page) * kPower;
                if (kPower == 4)
                    *(uint32_t*)y = *(const uint32_t*)x;
                else
                    *(uint16_t*)y = *(const uint16_t*)x;
            }
        }
        return;
    }
    if (part) return;
    // Where token old[u] is and its place u, for kDeep of them: blocks and rows of a head. False: nothing to move.
    struct Move {
        int32_t block, to_block;
        uint32_t slot, to_slot;
    };
    auto find = [&](int32_t i, int32_t old, Move& m) {
        if (old < 0 || !locate(p, from, old, m.block, m.slot) || !locate(p, to, i, m.to_block, m.to_slot)) return false;
        return m.block != m.to_block || m.slot != m.to_slot;
    };
    if (kind == planes * slices) {  // the weights
        const int32_t per = kMoveThreads * kDeep;
        for (int32_t i0 = 0; i0 < k.m; i0 += per) {
            int32_t old[kDeep];
            float x[kDeep];
            float* at[kDeep];
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                const int32_t i = i0 + u * kMoveThreads + threadIdx.x;
                old[u] = i < k.m ? source[i] : -1;
            }
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                Move m;
                at[u] = nullptr;
                if (!find(i0 + u * kMoveThreads + threadIdx.x, old[u], m)) continue;
                x[u] = *weight_at(p, layer, head, m.block, m.slot);
                at[u] = weight_at(p, layer, head, m.to_block, m.to_slot);
            }
            arrive<0>();
            __syncthreads();  // the chunk is read
#pragma unroll
            for (int u = 0; u < kDeep; ++u)
                if (at[u]) *at[u] = x[u];
        }
        return;
    }
    const int plane = kind % planes, slice = kind / planes;
    uint8_t* const base = (plane ? p.v : p.k) + (int64_t)layer * p.layer;
    // a lane moves piece `column` of every `per`th row
    const int lanes = columns < kSlice ? columns : kSlice, per = kMoveThreads / lanes;
    const int column = slice * kSlice + threadIdx.x % lanes, line = threadIdx.x / lanes;
    const bool power = kPower && column == 0;
    const int32_t chunk = per * kDeep;
    int32_t old[kDeep];
    auto look = [&](int32_t i0) {
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            const int32_t i = i0 + u * per + line;
            old[u] = i < k.m ? source[i] : -1;
        }
    };
    look(0);
    for (int32_t i0 = 0; i0 < k.m; i0 += chunk) {
        v4u x[kDeep];
        uint32_t e[kDeep];
        uint8_t* at[kDeep];  // where a row goes, or null
        uint8_t* power_at[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            Move m;
            at[u] = nullptr;
            if (!find(i0 + u * per + line, old[u], m)) continue;
            const int64_t row = (int64_t)head * p.div.page + m.slot, to_row = (int64_t)head * p.div.page + m.to_slot;
            uint8_t* const slab = base + (int64_t)m.block * p.slab;
            uint8_t* const to_slab = base + (int64_t)m.to_block * p.slab;
            at[u] = to_slab + to_row * p.row + column * 16;
            x[u] = __builtin_nontemporal_load((const v4u*)(slab + row * p.row + column * 16));
            if (power) {
                power_at[u] = to_slab + p.powers + to_row * kPower;
                const uint8_t* const y = slab + p.powers + row * kPower;
                e[u] = kPower == 4 ? *(const uint32_t*)y : *(const uint16_t*)y;
            }
        }
        look(i0 + chunk);  // the next chunk's tokens
        arrive<0>();
        __syncthreads();  // the chunk is read
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            if (!at[u]) continue;
            __builtin_nontemporal_store(x[u], (v4u*)at[u]);
            if (power) {
                if (kPower == 4)
                    *(uint32_t*)power_at[u] = e[u];
                else
                    *(uint16_t*)power_at[u] = (uint16_t)e[u];
            }
        }
    }
}

int columns_of(const KeepPlan& p) { return p.row / 16; }
int slices_of(const KeepPlan& p) { return (columns_of(p) + kSlice - 1) / kSlice; }

}  // namespace

int64_t keep_workgroups(const KeepPlan& p) {
    return (int64_t)p.layers * p.R * p.heads * ((p.v ? 2 : 1) * slices_of(p) + 1);
}

hipError_t launch_keep(const KeepPlan& p, int cus, hipStream_t s) {
    const int64_t units = (int64_t)p.layers * p.R * p.heads;
    hipLaunchKernelGGL(k_keep_select, dim3((unsigned)units), dim3(kSelectThreads), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int planes = p.v ? 2 : 1, slices = slices_of(p), columns = columns_of(p);
    const PageDiv pieces = page_div(planes * columns);
    const int64_t want = (int64_t)kMovers * cus / keep_workgroups(p);
    const int kinds = planes * slices + 1;
    const int64_t most = ((int64_t)p.max_keep + kinds * kTokens - 1) / (kinds * kTokens);  // that have tokens to move
    int parts = want < 1 ? 1 : want < kMostParts ? (int)want : kMostParts;
    if (parts > most) parts = most < 1 ? 1 : (int)most;
    const dim3 grid((unsigned)(keep_workgroups(p) * parts));
    if (p.power == 4)
        hipLaunchKernelGGL(k_keep_move<4>, grid, dim3(kMoveThreads), 0, s, p, planes, slices, columns, parts, pieces);
    else if (p.power == 2)
        hipLaunchKernelGGL(k_keep_move<2>, grid, dim3(kMoveThreads), 0, s, p, planes, slices, columns, parts, pieces);
    else
        hipLaunchKernelGGL(k_keep_move<0>, grid, dim3(kMoveThreads), 0, s, p, planes, slices, columns, parts, pieces);
    return hipGetLastError();
}

}  // namespace ptsd
