// Block tables, slot maps and positions from a batch's request lengths.
//
// Request r, with held_r blocks, past_r tokens and n_r new ones, wants
// ceil((past_r + n_r) / page) - held_r more blocks. Its first is entry
// first + (the wants of the requests before it) of the free list: one prefix
// sum over the batch. Then every new table entry and every token's slot is a
// search for its request and two loads.
//
// The work is a few bytes a token, so what counts is latency: one launch, no
// workspace and no flags between workgroups. A workgroup sums the wants before
// its chunk of requests for itself (16 bytes a request, from L2) and scans the
// chunk's own in LDS; `parts` workgroups of a chunk share its entries and tokens.
// 1 request of 1,000 tokens takes 4.4 us, 256 of one token 6.6, 700 of 1 to 2,801 (980,000
// tokens, 12 MB written) 9.7: its writes alone would take 2 us, the rest are the
// dependent trips lengths, sum, search, free entry, slot.
#include <hip/hip_runtime.h>

#include "paged.hpp"

namespace ptsd {
namespace {

constexpr int kThreads = 512;
constexpr int kChunk = 1024;             // requests a workgroup scans
constexpr int kPer = kChunk / kThreads;  // consecutive ones a thread
constexpr int kTokensPer = 4;            // consecutive tokens a thread's step

typedef long long v2l __attribute__((ext_vector_type(2)));
typedef int v4i __attribute__((ext_vector_type(4)));

struct Request {
    int64_t begin, end;  // tokens of the batch
    int64_t past;
    int32_t held, want;
};

__device__ Request request(const TablesPlan& p, int r) {
    Request q;
    const int64_t a = p.offsets[r], b = p.offsets[r + 1];
    const bool ok = a >= 0 && b >= a && b <= p.n_tokens;
    q.begin = a;
    q.end = ok ? b : a;  // a malformed request has no tokens
    q.past = p.context[r];
    int held = p.held ? p.held[r] : 0;
    held = held < 0 ? 0 : (held > p.max_blocks ? p.max_blocks : held);
    q.held = held;
    const int64_t room = (int64_t)p.max_blocks * p.div.page;  // at most 2^30
    int64_t tokens = q.past + (q.end - q.begin);
    tokens = tokens < 0 ? 0 : (tokens > room ? room : tokens);
    const int32_t need = (int32_t)div_page((uint32_t)tokens + p.div.page - 1, p.div);
    q.want = need > held ? need - held : 0;
    return q;
}

// Sum over the workgroup; every thread gets it.
__device__ int32_t sum_all(int32_t x, int32_t* part) {
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    int32_t t = 0;
    for (int w = 0; w < kThreads / 64; ++w) t += part[w];
    return t;
}

__global__ __launch_bounds__(kThreads) void k_tables(TablesPlan p, int parts) {
    // the chunk's requests: tokens, first token's position, blocks held, wanted before
    __shared__ int64_t s_begin[kChunk], s_end[kChunk];
    __shared__ int32_t s_past[kChunk], s_held[kChunk], s_want[kChunk + 1];
    __shared__ int32_t s_part[kThreads / 64];
    const int tid = threadIdx.x;
    const int chunk = blockIdx.x / parts, part = blockIdx.x % parts;
    const int r0 = chunk * kChunk;
    const int nr = p.R - r0 < kChunk ? p.R - r0 : kChunk;

    // R * max_blocks <= 2^29, so every sum of wants fits 32 bits
    int32_t before = 0;
    for (int r = tid; r < r0; r += kThreads) before += request(p, r).want;
    if (r0) before = sum_all(before, s_part);

    int32_t want[kPer], mine = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int l = tid * kPer + i;
        want[i] = 0;
        if (l < nr) {
            const Request q = request(p, r0 + l);
            want[i] = q.want;
            s_begin[l] = q.begin;
            s_end[l] = q.end;
            s_past[l] = (int32_t)q.past;
            s_held[l] = q.held;
        }
        mine += want[i];
    }
    int32_t scan = mine;  // inclusive over the wave
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t o = __shfl_up(scan, d);
        if ((tid & 63) >= d) scan += o;
    }
    __syncthreads();
    if ((tid & 63) == 63) s_part[tid >> 6] = scan;
    __syncthreads();
    int32_t at = scan - mine;
    for (int w = 0; w < (tid >> 6); ++w) at += s_part[w];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (tid * kPer + i <= nr) s_want[tid * kPer + i] = at;
        at += want[i];
    }
    if (tid == kThreads - 1) s_want[nr] = at;
    __syncthreads();

    int64_t first = p.first ? *p.first : 0;
    if (first < 0) first = 0;
    const int64_t avail = p.n_free > first ? p.n_free - first : 0;
    const int32_t total = s_want[nr];
    // of them this chunk's wants get the first `left`: `first` may be any number, so it is added
    // only for those
    const int64_t left = avail - before;

    if (part == 0) {
        for (int l = tid; l < nr; l += kThreads) {
            const int64_t rest = left - s_want[l];
            const int32_t w = s_want[l + 1] - s_want[l];
            const int64_t given = rest < 0 ? 0 : (rest < w ? rest : w);
            p.held_out[r0 + l] = s_held[l] + (int32_t)given;
        }
        if (tid == 0 && r0 + nr == p.R) {
            const int64_t all = (int64_t)before + total;
            *p.next = first + (all < avail ? all : avail);
        }
    }

    const int64_t step = (int64_t)parts * kThreads;
    for (int64_t e = (int64_t)part * kThreads + tid; e < total; e += step) {
        int lo = 0, hi = nr - 1;  // the last request that starts at or before e
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (s_want[mid] <= e)
                lo = mid;
            else
                hi = mid - 1;
        }
        p.table[(int64_t)(r0 + lo) * p.max_blocks + s_held[lo] + (e - s_want[lo])] =
            e < left ? p.free_blocks[first + before + e] : -1;
    }

    // tokens of the chunk: [the first request's first, the next chunk's first);
    // those before the first chunk and behind the last belong to no request
    int64_t t0 = chunk ? p.offsets[r0] : 0;
    int64_t t1 = r0 + nr < p.R ? p.offsets[r0 + nr] : p.n_tokens;
    if (t0 < 0) t0 = 0;
    if (t1 > p.n_tokens) t1 = p.n_tokens;
    const int64_t room = (int64_t)p.max_blocks * p.div.page;
    // groups of four tokens by their number, so that they are written as one where the
    // arrays are aligned
    const bool whole = ((reinterpret_cast<uintptr_t>(p.slots) | reinterpret_cast<uintptr_t>(p.positions)) & 15) == 0;
    for (int64_t t = t0 / kTokensPer * kTokensPer + ((int64_t)part * kThreads + tid) * kTokensPer; t < t1;
         t += step * kTokensPer) {
        int lo = 0, hi = nr - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (s_begin[mid] <= t)
                lo = mid;
            else
                hi = mid - 1;
        }
        int64_t slot[kTokensPer];
        int32_t pos[kTokensPer];
#pragma unroll
        for (int i = 0; i < kTokensPer; ++i) {
            const int64_t ti = t + i;
            slot[i] = -1;
            pos[i] = 0;
            while (lo + 1 < nr && s_begin[lo + 1] <= ti) ++lo;
            if (nr == 0 || ti < s_begin[lo] || ti >= s_end[lo]) continue;
            const int64_t at_pos = s_past[lo] + (ti - s_begin[lo]);
            pos[i] = (int32_t)at_pos;
            if (at_pos < 0 || at_pos >= room) continue;
            const uint32_t b = div_page((uint32_t)at_pos, p.div);
            int64_t entry;
            if ((int32_t)b < s_held[lo]) {
                entry = p.table[(int64_t)(r0 + lo) * p.max_blocks + b];
            } else {
                const int32_t e = s_want[lo] + ((int32_t)b - s_held[lo]);
                entry = e < left ? p.free_blocks[first + before + e] : -1;
            }
            if (entry >= 0) slot[i] = entry * p.div.page + ((uint32_t)at_pos - b * p.div.page);
        }
        if (whole && t >= t0 && t + kTokensPer <= t1) {
            *(v2l*)(p.slots + t) = v2l{slot[0], slot[1]};
            *(v2l*)(p.slots + t + 2) = v2l{slot[2], slot[3]};
            if (p.positions) *(v4i*)(p.positions + t) = v4i{pos[0], pos[1], pos[2], pos[3]};
        } else {
#pragma unroll
            for (int i = 0; i < kTokensPer; ++i) {
                if (t + i < t0 || t + i >= t1) continue;
                p.slots[t + i] = slot[i];
                if (p.positions) p.positions[t + i] = pos[i];
            }
        }
    }
}

}  // namespace

hipError_t launch_tables(const TablesPlan& p, hipStream_t s) {
    const int chunks = p.R > 0 ? (p.R + kChunk - 1) / kChunk : 1;  // without requests: `next` alone
    // a part for every step of the tokens, up to about two workgroups a compute unit
    int64_t parts = (p.n_tokens / chunks + kThreads * kTokensPer - 1) / (kThreads * kTokensPer);
    const int64_t most = chunks < 512 ? 512 / chunks : 1;
    parts = parts < 1 ? 1 : (parts > most ? most : parts);
    hipLaunchKernelGGL(k_tables, dim3((unsigned)(chunks * parts)), dim3(kThreads), 0, s, p, (int)parts);
    return hipGetLastError();
}

}  // namespace ptsd
