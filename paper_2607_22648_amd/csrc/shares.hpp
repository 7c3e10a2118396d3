// A batch's work in equal shares (decode.hip, latent_attend.hip): the steps of keys of all requests
// and tiles of query rows, laid end to end, one share for each workgroup that the device holds. A
// plan has offsets, context, n_tokens, R, max_blocks, the page division, the rows of a token (group)
// and few_rows, the most rows of a request that count.
#pragma once

#include <hip/hip_runtime.h>

#include "paged.hpp"

namespace ptsd {

// A request's work for a KV head: its steps of keys for each of its tiles. A
// request that sees no key has one step, which writes its zeros.
struct Work {
    int64_t begin;  // first token
    int32_t n;
    int64_t past;
    int32_t steps, tiles;
    __device__ int64_t all() const { return (int64_t)steps * tiles; }
};

// kSpare: steps without keys at each tile's end, for what a tile takes beside its keys: equal shares of short
// requests would last longer.
template <int kRows, int kSpare = 0, class Plan>
__device__ inline Work work_of(const Plan& p, int r, int step_keys) {
    Work w;
    const int64_t a = p.offsets[r], b = p.offsets[r + 1];
    const bool ok = a >= 0 && b > a && b <= p.n_tokens && (b - a) * p.group <= p.few_rows;
    w.begin = ok ? a : 0;
    w.n = ok ? (int32_t)(b - a) : 0;
    w.past = p.context[r];
    const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
    int64_t end = w.past + w.n;
    end = end < 1 ? 1 : (end > limit ? limit : end);
    w.steps = (int32_t)((end + step_keys - 1) / step_keys) + kSpare;
    w.tiles = (w.n * p.group + kRows - 1) / kRows;
    return w;
}

// The shares: share w of `count` has steps [w all / count, (w + 1) all / count).
struct Shares {
    int64_t all, count;
    __device__ int64_t begin(int64_t w) const { return divided(w * all, count); }
    // the share that has step x: the last that begins at or before it
    __device__ int64_t of(int64_t x) const { return divided((x + 1) * count + all - 1, all) - 1; }
    // (a division of 64 bits takes a microsecond)
    static __device__ int64_t divided(int64_t a, int64_t b) {
        return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
    }
};

// Sums the batch's work, `of(r)` for each request, and finds the request `r` that the first (or last) step of
// share `share` of `count` is in, its work and its first step. Every workgroup does so for
// itself: thread t takes the requests from t ceil(R / threads) on. kLeast: steps of a share, of a batch of few.
template <int kWavesOf, int kLeast = 1, class W, class Of>
__device__ inline Shares find_share(int R, int64_t count, const Of& of, int64_t share, bool last, int& r, W& f,
                                    int64_t& first) {
    __shared__ int64_t s_sum[kWavesOf], s_first;
    __shared__ int s_r;
    __shared__ W s_work;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per = (R + kWavesOf * 64 - 1) / (kWavesOf * 64);
    const int r0 = threadIdx.x * per;
    W w;
    int64_t mine = 0;
    for (int i = 0; i < per && r0 + i < R; ++i) {
        w = of(r0 + i);
        mine += w.all();
    }
    int64_t scan = mine;
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t o = __shfl_up(scan, d);
        if (lane >= d) scan += o;
    }
    if (lane == 63) s_sum[wave] = scan;
    __syncthreads();
    Shares s{0, count};
    int64_t before = 0;
#pragma unroll
    for (int i = 0; i < kWavesOf; ++i) {
        if (i < wave) before += s_sum[i];
        s.all += s_sum[i];
    }
    if (s.all < s.count * kLeast) s.count = (s.all + kLeast - 1) / kLeast;
    const int64_t lo = before + scan - mine;
    const int64_t at = share >= s.count ? -1 : last ? s.begin(share + 1) - 1 : s.begin(share);
    if (at >= lo && at < lo + mine) {
        s_r = r0;
        s_first = lo;
        s_work = w;  // of the only request, if `per` is 1
    }
    __syncthreads();
    if (at < 0) return s;
    r = __builtin_amdgcn_readfirstlane(s_r);
    first = s_first;
    if (per == 1) {
        f = s_work;
        return s;
    }
    while (f = of(r), first + f.all() <= at) {
        first += f.all();
        ++r;
    }
    return s;
}

template <int kRows, int kWavesOf, int kSpare = 0, int kLeast = 1, class Plan>
__device__ inline Shares find_step(const Plan& p, int step_keys, int64_t share, bool last, int& r, Work& f,
                                   int64_t& first) {
    return find_share<kWavesOf, kLeast>(
        p.R, p.shares, [&](int i) { return work_of<kRows, kSpare>(p, i, step_keys); }, share, last, r, f, first);
}

}  // namespace ptsd
