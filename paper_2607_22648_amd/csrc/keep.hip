// Eviction: of each request, layer and KV head the most recent tokens stay, and of the others those of
// largest weight, ties by position. Their rows and weights move, in order, to the front of `to`.
//
// Two launches. The first finds what stays: a workgroup for each (layer, request, head) finds the
// weight from which on tokens stay by three passes over the weights' bits, 11, 11 and 10 at a time, counting
// them in LDS, and writes the positions in order; it moves the weights itself. The second moves the
// rows, bound by memory: what stays is read and written once.
//
// `to` may name the pages that the rows are on already. A row never moves back, so a workgroup that takes
// the rows of a unit in order, and has read a chunk whole before it writes it, overwrites nothing that is still to be
// read. A unit's planes, and 128 bytes of each row, are workgroups of their own.
#include <hip/hip_runtime.h>

#include "lds_fetch.hpp"
#include "weights.hpp"

namespace ptsd {
namespace {

typedef unsigned int v4u __attribute__((ext_vector_type(4)));

constexpr int kSelectThreads = 512;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 2048;
constexpr int kCached = 12288;  // weights that stay in LDS between passes; of longer requests they are read again
constexpr int kMoveThreads = 256;
constexpr int kSlice = 8;       // 16-byte pieces of a row that a workgroup moves
constexpr int kDeep = 8;        // rows of a lane under way

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

// Sums of all threads' values before a thread's, in thread order, and of all.
__device__ inline uint32_t scan(uint32_t x, uint32_t* s_wave, uint32_t& all) {
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
    all = 0;
#pragma unroll
    for (int i = 0; i < kSelectWaves; ++i) {
        if (i < wave) before += s_wave[i];
        all += s_wave[i];
    }
    return before + sum - x;
}

__global__ __launch_bounds__(kSelectThreads) void k_keep_select(KeepPlan p) {
    __shared__ uint32_t s_order[kCached];
    __shared__ uint32_t s_count[kBins];
    __shared__ uint32_t s_wave[kSelectWaves];
    __shared__ uint32_t s_bin, s_above;
    const int tid = threadIdx.x;
    const int unit = blockIdx.x, head = unit % p.heads, r = unit / p.heads % p.R, layer = unit / p.heads / p.R;
    const Kept k = kept_of(p, r);
    if (layer == 0 && head == 0 && tid == 0) p.context_out[r] = k.m;
    if (k.m == 0) return;
    const int32_t* const table = p.from + (int64_t)r * p.max_blocks;
    const int32_t* const to = p.to + (int64_t)r * p.max_blocks;
    int32_t* const source = p.source + (int64_t)unit * p.max_keep;
    const int32_t rest = k.n - k.recent;                   // candidates
    uint32_t want = (uint32_t)(k.m - k.recent);            // of them
    auto read = [&](int32_t i) {
        int32_t block;
        uint32_t slot;
        return locate(p, table, i, block, slot) ? order_of(*weight_at(p, layer, head, block, slot)) : 0u;
    };
    const bool cached = rest <= kCached, all_stay = (int32_t)want == rest, none = want == 0;
    uint32_t border = 0;  // tokens above it stay, and of those at it the first `want`
    if (!all_stay && !none) {
        for (int pass = 0; pass < 3; ++pass) {
            const int bits = pass < 2 ? 11 : 10, low = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            for (int b = tid; b < kBins; b += kSelectThreads) s_count[b] = 0;
            __syncthreads();
            for (int32_t i = tid; i < rest; i += kSelectThreads) {
                uint32_t x;
                if (pass == 0 || !cached) {
                    x = read(i);
                    if (cached) s_order[i] = x;
                } else {
                    x = s_order[i];
                }
                if (pass == 0 || x >> (low + bits) == border >> (low + bits))
                    atomicAdd(&s_count[(x >> low) & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
            // thread t has the bins 2047 - 4 t .. 2044 - 4 t: the largest first
            constexpr int kOf = kBins / kSelectThreads;
            uint32_t mine[kOf], sum = 0, total;
#pragma unroll
            for (int j = 0; j < kOf; ++j) {
                mine[j] = s_count[kBins - 1 - (tid * kOf + j)];
                sum += mine[j];
            }
            uint32_t above = scan(sum, s_wave, total);
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
    // In order: the positions that stay, and their weights.
    uint32_t done = 0, tied = 0;
    for (int32_t i0 = 0; i0 < k.n; i0 += kSelectThreads) {
        const int32_t i = i0 + tid;
        int32_t block = 0;
        uint32_t slot = 0;
        bool there = false;
        float weight = 0.f;
        if (i < k.n && (there = locate(p, table, i, block, slot))) weight = *weight_at(p, layer, head, block, slot);
        const uint32_t x = there ? order_of(weight) : 0u;
        const bool candidate = i < rest;
        bool stays = i < k.n && (!candidate || all_stay);
        if (!all_stay && !none) {
            const bool tie = candidate && x == border;
            uint32_t ties;
            const uint32_t rank = scan(tie, s_wave, ties);
            stays |= candidate && (x > border || (tie && tied + rank < want));
            tied += ties;
        }
        uint32_t some;
        const uint32_t at = done + scan(stays, s_wave, some);
        done += some;
        // all of the chunk's weights are read: the scan has waited for them
        if (stays) {
            source[at] = there ? i : -1;
            int32_t to_block;
            uint32_t to_slot;
            if (there && locate(p, to, (int32_t)at, to_block, to_slot)) *weight_at(p, layer, head, to_block, to_slot) = weight;
        }
        __syncthreads();
    }
}

// kPower: bytes of a row's exponents.
template <int kPower>
__global__ __launch_bounds__(kMoveThreads) void k_keep_move(KeepPlan p, int planes, int slices, int columns) {
    const int plane = blockIdx.x % planes, slice = blockIdx.x / planes % slices;
    const int unit = blockIdx.x / planes / slices;
    const int head = unit % p.heads, r = unit / p.heads % p.R, layer = unit / p.heads / p.R;
    const Kept k = kept_of(p, r);
    if (k.m == 0) return;
    const int32_t* const from = p.from + (int64_t)r * p.max_blocks;
    const int32_t* const to = p.to + (int64_t)r * p.max_blocks;
    const int32_t* const source = p.source + (int64_t)unit * p.max_keep;
    uint8_t* const base = (plane ? p.v : p.k) + (int64_t)layer * p.layer;
    // a lane moves piece `column` of every `per`th row
    const int lanes = columns < kSlice ? columns : kSlice, per = kMoveThreads / lanes;
    const int column = slice * kSlice + threadIdx.x % lanes, line = threadIdx.x / lanes;
    const bool power = kPower && column == 0;
    for (int32_t i0 = 0; i0 < k.m; i0 += per * kDeep) {
        v4u x[kDeep];
        uint32_t e[kDeep];
        int64_t at[kDeep];  // where it goes: a row of a slab's head, or -1
        int32_t old[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            const int32_t i = i0 + u * per + line;
            old[u] = i < k.m ? source[i] : -1;
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            const int32_t i = i0 + u * per + line;
            at[u] = -1;
            e[u] = 0;
            x[u] = v4u{0u, 0u, 0u, 0u};
            int32_t block, to_block;
            uint32_t slot, to_slot;
            if (old[u] < 0 || !locate(p, from, old[u], block, slot) || !locate(p, to, i, to_block, to_slot)) continue;
            if (block == to_block && slot == to_slot) continue;  // it is there already
            const int64_t row = (int64_t)head * p.div.page + slot;
            at[u] = (int64_t)to_block * p.slab + ((int64_t)head * p.div.page + to_slot) * p.row;
            x[u] = *(const v4u*)(base + (int64_t)block * p.slab + row * p.row + column * 16);
            if (power) {
                const uint8_t* const y = base + (int64_t)block * p.slab + p.powers + row * kPower;
                e[u] = kPower == 4 ? *(const uint32_t*)y : *(const uint16_t*)y;
            }
        }
        arrive<0>();
        __syncthreads();  // the chunk is read
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            if (at[u] < 0) continue;
            *(v4u*)(base + at[u] + column * 16) = x[u];
            if (power) {
                int32_t to_block;
                uint32_t to_slot;
                locate(p, to, i0 + u * per + line, to_block, to_slot);
                uint8_t* const y = base + (int64_t)to_block * p.slab + p.powers + ((int64_t)head * p.div.page + to_slot) * kPower;
                if (kPower == 4)
                    *(uint32_t*)y = e[u];
                else
                    *(uint16_t*)y = (uint16_t)e[u];
            }
        }
    }
}

int columns_of(const KeepPlan& p) { return p.row / 16; }
int slices_of(const KeepPlan& p) { return (columns_of(p) + kSlice - 1) / kSlice; }

}  // namespace

int64_t keep_workgroups(const KeepPlan& p) {
    return (int64_t)p.layers * p.R * p.heads * (p.v ? 2 : 1) * slices_of(p);
}

hipError_t launch_keep(const KeepPlan& p, hipStream_t s) {
    const int64_t units = (int64_t)p.layers * p.R * p.heads;
    hipLaunchKernelGGL(k_keep_select, dim3((unsigned)units), dim3(kSelectThreads), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)keep_workgroups(p));
    const int planes = p.v ? 2 : 1, slices = slices_of(p), columns = columns_of(p);
    if (p.power == 4)
        hipLaunchKernelGGL(k_keep_move<4>, grid, dim3(kMoveThreads), 0, s, p, planes, slices, columns);
    else if (p.power == 2)
        hipLaunchKernelGGL(k_keep_move<2>, grid, dim3(kMoveThreads), 0, s, p, planes, slices, columns);
    else
        hipLaunchKernelGGL(k_keep_move<0>, grid, dim3(kMoveThreads), 0, s, p, planes, slices, columns);
    return hipGetLastError();
}

}  // namespace ptsd
