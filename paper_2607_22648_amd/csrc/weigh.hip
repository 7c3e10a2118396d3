// The attention weights that a batch's queries gave to each cached token, added to what it had:
//   weight(j) += sum over rows that see key j of exp(scale q . k_j - lse).
//
// S = Q K^T, 32 x 32 at a time with keys as columns: a lane holds one key's scores of 16 rows, so that
// sums over rows stay in the lane, and no weight is ever rounded. Few rows are bound by reading K once;
// many by the matrix units and the exponentials (16 cycles of a wave for 64, as long as
// 2 dim operations of 32 rows take for dim 128), which two waves a SIMD overlap.
//
// A workgroup of four waves takes a tile of keys, 64 a wave (32 of a latent cache), as registers of the
// second factor, and goes through the query rows that see it, 32 at a time, which pass through LDS for
// all four. (Key tile, 32 rows) items of the batch, those above the diagonal left out, are laid end to end and
// cut into equal shares, as decode.hip's steps; a tile of more than 16 items may be cut, and a second kernel
// adds what its shares found, in order: the same inputs give the same bits.
#include "attend.hpp"
#include "lds_fetch.hpp"
#include "shares.hpp"
#include "weights.hpp"

namespace ptsd {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kRowsOf = 32;  // query rows of an item
constexpr int kWhole = 16;   // items of a tile that is not cut
constexpr int kLatent = 2;   // kinds of keys: 16 bits, 4 bits, latent rows

constexpr int keys_of(int layout) { return kWaves * (layout == kLatent ? 32 : 64); }  // of a tile

// A request's items. Its key tiles 0 .. seen + 1 - 1 are seen by all row tiles; tile seen + i by those from
// i * rise - late on (i >= 1): a tile's keys are a whole number of row tiles.
struct Items {
    int64_t begin;  // first token that has a position
    int32_t n;
    int32_t past;
    int32_t tiles, rows, seen;
    int64_t rise, late;
    // items before tile t
    __device__ int64_t before(int64_t t) const {
        const int64_t j = t - 1 - seen;
        return t * rows - (j > 0 ? rise * (j * (j + 1) / 2) - late * j : 0);
    }
    __device__ int64_t all() const { return before(tiles); }
    __device__ int32_t first_row(int32_t t) const {
        const int64_t i = t - seen;
        return i > 0 ? (int32_t)(i * rise - late) : 0;
    }
};

__device__ inline Items items_of(const WeighPlan& p, int r, int keys) {
    Items w;
    int64_t a = p.offsets[r], b = p.offsets[r + 1];
    const bool ok = a >= 0 && b > a && b <= p.n_tokens;
    int64_t past = p.context[r];
    if (past < 0) {  // tokens before position 0 see nothing
        a -= past;
        past = 0;
    }
    w.begin = a;
    w.n = ok && b > a ? (int32_t)(b - a) : 0;
    w.past = (int32_t)past;
    const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
    int64_t end = past + w.n;
    end = w.n == 0 ? 0 : end > limit ? limit : end;
    w.tiles = (int32_t)((end + keys - 1) / keys);
    w.rows = (int32_t)(((int64_t)w.n * p.group + kRowsOf - 1) / kRowsOf);
    w.seen = (int32_t)(past / keys);
    w.rise = (int64_t)(keys / kRowsOf) * p.group;
    w.late = (past % keys * p.group + kRowsOf - 1) / kRowsOf;
    return w;
}

// The tile that item y is in.
__device__ inline int32_t tile_of(const Items& f, int64_t y) {
    int32_t lo = 0, span = f.tiles;
    while (span > 1) {
        const int32_t half = span / 2;
        if (f.before(lo + half) <= y) {
            lo += half;
            span -= half;
        } else {
            span = half;
        }
    }
    return lo;
}

// A key's slot of the weights, or -1.
__device__ inline int64_t weight_at(const WeighPlan& p, int r, int head, int64_t key) {
    const uint32_t column = div_page((uint32_t)key, p.kv.div);
    const int32_t entry = p.table[(int64_t)r * p.max_blocks + column];
    if (entry < 0 || entry >= p.kv.blocks) return -1;
    return ((int64_t)entry * p.kv.heads + head) * p.kv.div.page + ((uint32_t)key - column * p.kv.div.page);
}

__device__ inline void put_weight(const WeighPlan& p, int r, int head, int32_t key, float sum) {
    const int64_t at = weight_at(p, r, head, key);
    if (at < 0) return;
    const int32_t had = p.weighed ? p.weighed[r] : p.context[r];
    p.weights[at] = key < had ? p.weights[at] + sum : sum;
}

// kDim: of a row; kLayout: how keys are kept.
template <int kDim, bool kHalf, int kLayout>
__global__ __launch_bounds__(kThreads, 2) void k_weigh(WeighPlan p) {
    using E = Elem<kHalf>;
    using V8 = typename E::v8;
    constexpr bool kFour = kLayout == 1;
    constexpr int kTile = keys_of(kLayout), kChunks = kTile / kWaves / 32;
    constexpr int kSteps = kDim / 16, kColumns = kDim / 8;  // matrix steps; 16-byte columns of a row
    // Of a row, or of each part of a latent one, a lane takes half, so that whole lines are read: queries in LDS
    // likewise. Rows in LDS are padded by a column, so that 16 lanes which read one column of 16 rows find 16
    // places; the shared parts of latent queries, which come eight rows to a load, are turned instead.
    constexpr int kOwn = kLayout == kLatent ? kSteps - kRope / 16 : kSteps;  // steps before the shared part
    constexpr int kRow = kOwn * 32 + 16, kRopeRow = kRope * 2;
    constexpr int kPieces = kLayout == kLatent ? 1 : kRowsOf * kColumns / kThreads;  // of queries, a thread
    constexpr int kBuffer = kRowsOf * (kRow + (kLayout == kLatent ? kRopeRow : 0));
    __shared__ __attribute__((aligned(16))) uint8_t s_q[2][kBuffer];
    __shared__ float s_lse[2][kRowsOf];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int head = blockIdx.x % p.kv.heads, share = blockIdx.x / p.kv.heads;
    int r;
    int64_t first;
    Items f;
    const Shares shares = find_share<kWaves>(
        p.R, p.shares, [&](int i) { return items_of(p, i, kTile); }, share, false, r, f, first);
    if (share >= shares.count) return;
    const int64_t share0 = shares.begin(share), share1 = shares.begin(share + 1);
    for (int64_t done = share0; done < share1;) {
        while (done >= first + f.all()) {
            first += f.all();
            f = items_of(p, ++r, kTile);
        }
        const int32_t tile = tile_of(f, done - first);
        const int64_t tile0 = first + f.before(tile), tile1 = first + f.before(tile + 1);
        if (f.rows <= kWhole && done > tile0) {  // the share before has all of it
            done = tile1;
            continue;
        }
        const int32_t row_first = f.first_row(tile);
        const int32_t rt0 = row_first + (int32_t)(done - tile0);
        const int64_t stop = f.rows <= kWhole || tile1 < share1 ? tile1 : share1;
        const int32_t rt1 = row_first + (int32_t)(stop - tile0);
        const bool part = done > tile0 || stop < tile1;
        float* const to = p.parts + (2 * (int64_t)blockIdx.x + (done > tile0 ? 0 : 1)) * kTile;
        done = stop;

        const int64_t limit64 = (int64_t)p.max_blocks * p.kv.div.page;
        const int64_t end64 = (int64_t)f.past + f.n < limit64 ? (int64_t)f.past + f.n : limit64;
        const int32_t end = (int32_t)end64;
        const int32_t k0 = tile * kTile + wave * (32 * kChunks);
        const int all_rows = f.n * p.group;
        const int32_t* const table = p.table + (int64_t)r * p.max_blocks;

        // keys: column n, kSteps columns of 8 values a lane
        V8 k[kChunks][kSteps];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int32_t key = k0 + 32 * c + n, last = end - 1;
            const int32_t entry = table[div_page((uint32_t)(key < last ? key : last), p.kv.div)];
            const bool there = key < end && entry >= 0 && entry < (int32_t)p.kv.blocks;
            const uint32_t block = there ? (uint32_t)entry : 0u;
            const uint32_t slot = there ? (uint32_t)key - div_page((uint32_t)key, p.kv.div) * p.kv.div.page : 0u;
            if constexpr (kLayout == kLatent) {
                const uint8_t* row = p.latent.rows + ((uint64_t)((block * p.kv.div.page + slot) * p.latent.line) << 4);
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
                    k[c][i] = __builtin_bit_cast(V8, *(const v4u*)(row + (i < kOwn ? i + kOwn * half : i + kOwn + (kSteps - kOwn) * half) * 16));
            } else {
                const uint32_t line = head * p.kv.div.page + slot;
                if constexpr (kFour) {
                    const uint8_t* row = p.kv.k + (uint64_t)block * p.kv.slab + (uint64_t)line * (kDim / 2) + half * (kDim / 4);
                    const uint8_t* power = p.kv.k + (uint64_t)block * p.kv.slab + p.kv.exponents +
                                           (uint64_t)line * (kDim / kGroup) + half * (kDim / 2 / kGroup);
#pragma unroll
                    for (int g = 0; g < kSteps / 4; ++g) {
                        const v4u codes = *(const v4u*)(row + g * 16);
                        const float step = step_of(power[g]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) k[c][4 * g + i] = __builtin_bit_cast(V8, widen8(codes[i], step));
                    }
                } else {
                    const uint8_t* row = p.kv.k + (uint64_t)block * p.kv.slab + (uint64_t)line * (kDim * 2) + half * kDim;
#pragma unroll
                    for (int i = 0; i < kSteps; ++i) k[c][i] = __builtin_bit_cast(V8, *(const v4u*)(row + i * 16));
                }
            }
        }

        v4u piece[kPieces];
        float lse = 0.f;
        // a tile of query rows on its way to LDS, by registers, a latent cache's straight there (its rows would take
        // 36 registers); rows past the last one as the last
        auto load = [&](int rt, int buffer) {
            auto place = [&](int j, int& token, int& sub) {
                const int row = rt * kRowsOf + j < all_rows ? rt * kRowsOf + j : all_rows - 1;
                token = row / p.group;
                sub = row - token * p.group;
            };
            int token, sub;
            if constexpr (kLayout == kLatent) {
                place(n, token, sub);
                const int64_t own = (f.begin + token) * p.q.token + (int64_t)sub * p.q.head;
                const int64_t shared = (f.begin + token) * p.qr.token + (int64_t)sub * p.qr.head;
                const uint32_t to = lds_of(s_q[buffer]);
#pragma unroll
                for (int i = 0; i < kRowsOf / kWaves; ++i) {
                    const int j = wave * (kRowsOf / kWaves) + i;
                    const int64_t at = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)own, j) |
                                       (int64_t)__builtin_amdgcn_readlane((int)(own >> 32), j) << 32;
                    if (lane < kOwn * 2) fetch16((const uint8_t*)p.q.p + at * 2, (uint32_t)lane * 16, to + j * kRow);
                }
                const int j = wave * 8 + (lane >> 3);
                const int64_t at = (int64_t)(uint32_t)__builtin_amdgcn_ds_bpermute(4 * j, (int)shared) |
                                   (int64_t)__builtin_amdgcn_ds_bpermute(4 * j, (int)(shared >> 32)) << 32;
                fetch16_at((const uint8_t*)p.qr.p + at * 2 + ((lane & 7) ^ ((j >> 1) & 7)) * 16,
                           to + kRowsOf * kRow + wave * 8 * kRopeRow);
            } else {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int at = threadIdx.x + i * kThreads, c = at % kColumns;
                    place(at / kColumns, token, sub);
                    piece[i] = *(const v4u*)((const uint8_t*)p.q.p + ((f.begin + token) * p.q.token +
                                                                     (int64_t)(head * p.group + sub) * p.q.head) * 2 + c * 16);
                }
            }
            if (threadIdx.x < kRowsOf) {
                place(threadIdx.x, token, sub);
                lse = rt * kRowsOf + (int)threadIdx.x < all_rows
                          ? p.lse[(f.begin + token) * p.q_heads + head * p.group + sub] : -INFINITY;
                // rows that saw no key, and those that do not exist, give nothing: a weight of 2^-inf
                lse = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f;
            }
        };
        auto store = [&](int buffer) {
            if constexpr (kLayout != kLatent) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int at = threadIdx.x + i * kThreads, j = at / kColumns, c = at % kColumns;
                    *(v4u*)(s_q[buffer] + j * kRow + c * 16) = piece[i];
                }
            }
            if (threadIdx.x < kRowsOf) s_lse[buffer][threadIdx.x] = lse;
            arrive<0>();
        };

        float total[kChunks], sum[kChunks];  // sums of sums: an error of few of them, not of all
#pragma unroll
        for (int c = 0; c < kChunks; ++c) total[c] = sum[c] = 0.f;
        __syncthreads();  // all are done with the tile before
        load(rt0, 0);
        store(0);
        __syncthreads();
        for (int32_t rt = rt0; rt < rt1; ++rt) {
            const int buffer = (rt - rt0) & 1;
            if (rt + 1 < rt1) load(rt + 1, buffer ^ 1);
            const uint8_t* const mem = s_q[buffer] + n * kRow + half * (kOwn * 16);
            v16f s[kChunks];
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[c][e] = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const uint8_t* const at = i < kOwn ? mem + i * 16
                                                   : s_q[buffer] + kRowsOf * kRow + n * kRopeRow +
                                                         ((i - kOwn + (kSteps - kOwn) * half) ^ ((n >> 1) & 7)) * 16;
                const V8 q = __builtin_bit_cast(V8, *(const v4u*)at);
#pragma unroll
                for (int c = 0; c < kChunks; ++c) s[c] = E::mma32(q, k[c][i], s[c]);
            }
            // rows 8 (e >> 2) + 4 half + (e & 3) in s[..][e]
            const int64_t sees = (int64_t)f.past + rt * kRowsOf / p.group;  // the first row's last key
            const bool edge = k0 + 32 * kChunks - 1 > sees;
            float weight[kChunks] = {};
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const v4f less = *(const v4f*)&s_lse[buffer][8 * a + 4 * half];
                float w[kChunks][4];
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[c][e] = exp2_of(__builtin_fmaf(s[c][4 * a + e], p.scale2, -less[e]));
                if (edge) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int row = rt * kRowsOf + 8 * a + 4 * half + e;
                        const int64_t pos = (int64_t)f.past + row / p.group;
#pragma unroll
                        for (int c = 0; c < kChunks; ++c)
                            if (k0 + 32 * c + n > pos) w[c][e] = 0.f;
                    }
                }
#pragma unroll
                for (int c = 0; c < kChunks; ++c) weight[c] += (w[c][0] + w[c][1]) + (w[c][2] + w[c][3]);
            }
#pragma unroll
            for (int c = 0; c < kChunks; ++c) sum[c] += weight[c];
            if (((rt - rt0) & 31) == 31) {
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    total[c] += sum[c];
                    sum[c] = 0.f;
                }
            }
            if (rt + 1 < rt1) store(buffer ^ 1);
            __syncthreads();
        }
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            total[c] += sum[c];
            total[c] += __shfl_xor(total[c], 32);
            const int in_tile = (wave * kChunks + c) * 32 + n;
            if (half) continue;
            if (part)
                to[in_tile] = total[c];
            else if (tile * kTile + in_tile < end)
                put_weight(p, r, head, tile * kTile + in_tile, total[c]);
        }
    }
}

// Adds the parts of tiles that several shares have: the workgroup of the share that begins a tile does.
template <int kLayout>
__global__ __launch_bounds__(keys_of(kLayout)) void k_weigh_join(WeighPlan p) {
    constexpr int kTile = keys_of(kLayout);
    const int head = blockIdx.x % p.kv.heads, share = blockIdx.x / p.kv.heads;
    int r;
    int64_t first;
    Items f;
    const Shares shares = find_share<kTile / 64>(
        p.R, p.shares, [&](int i) { return items_of(p, i, kTile); }, share, true, r, f, first);
    if (share >= shares.count || f.rows <= kWhole) return;
    const int64_t share0 = shares.begin(share), share1 = shares.begin(share + 1);
    const int32_t tile = tile_of(f, share1 - 1 - first);
    const int64_t tile0 = first + f.before(tile), tile1 = first + f.before(tile + 1);
    if (tile0 < share0 || tile1 <= share1) return;
    const int64_t last = shares.of(tile1 - 1);
    const int64_t step = 2 * (int64_t)p.kv.heads * kTile;
    const float* from = p.parts + (2 * (int64_t)blockIdx.x + 1) * kTile + threadIdx.x;
    float sum = *from;
    from += step - kTile;  // the first part of the next share
#pragma unroll 8
    for (int64_t i = share + 1; i <= last; ++i, from += step) sum += *from;
    const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
    const int64_t end = (int64_t)f.past + f.n < limit ? (int64_t)f.past + f.n : limit;
    const int64_t key = (int64_t)tile * kTile + threadIdx.x;
    if (key < end) put_weight(p, r, head, (int32_t)key, sum);
}

template <int kDim, bool kHalf, int kLayout>
hipError_t run(const WeighPlan& p, hipStream_t s) {
    const dim3 grid((unsigned)(p.shares * p.kv.heads));
    hipLaunchKernelGGL((k_weigh<kDim, kHalf, kLayout>), grid, dim3(kThreads), 0, s, p);
    const hipError_t e = hipGetLastError();
    // no request can have a tile that is cut
    if (e != hipSuccess || p.n_tokens * p.group <= kWhole * kRowsOf) return e;
    hipLaunchKernelGGL((k_weigh_join<kLayout>), grid, dim3(keys_of(kLayout)), 0, s, p);
    return hipGetLastError();
}

template <int kDim>
hipError_t run_kind(const WeighPlan& p, hipStream_t s) {
    if (p.kv.kind == PTSTORE_KV_MXFP4) return run<kDim, false, 1>(p, s);
    return p.kv.kind == PTSTORE_KV_FP16 ? run<kDim, true, 0>(p, s) : run<kDim, false, 0>(p, s);
}

template <int kDim>
hipError_t run_latent(const WeighPlan& p, hipStream_t s) {
    return p.latent.kind == PTSTORE_KV_FP16 ? run<kDim, true, kLatent>(p, s) : run<kDim, false, kLatent>(p, s);
}

}  // namespace

// As many workgroups as fill the device: four a compute unit.
int weigh_shares(int32_t heads, int cus) {
    const int shares = 4 * cus / heads;
    return shares > 0 ? shares : 1;
}

int64_t weigh_workspace(int32_t heads, int cus) {
    return 2ll * weigh_shares(heads, cus) * heads * keys_of(0) * (int64_t)sizeof(float);
}

hipError_t launch_weigh(const WeighPlan& p, hipStream_t s) {
    if (p.is_latent) return p.latent.latent == 512 ? run_latent<512 + kRope>(p, s) : run_latent<256 + kRope>(p, s);
    return p.kv.dim == 128 ? run_kind<128>(p, s) : run_kind<64>(p, s);
}

}  // namespace ptsd
