// New tokens' K and V into their pages, and rows of pages back out.
//
// 16-bit caches: a copy, 16 bytes a lane, consecutive lanes along a row.
//
// 4-bit caches: 32 elements share the exponent e, the smallest with
// max |x| <= 7 * 2^e, and each is stored as the 4-bit float (levels 0, 1/2, 1,
// 3/2, 2, 3, 4, 6) nearest to x / 2^e, ties to the even code. A value between
// 6 and 7 steps becomes 6, an error of at most one step, which is what the
// widest gap (4 to 6) costs anyway; the next exponent would double it for all
// 32. A power of two divides without rounding, so codes and what they stand
// for are exact in every precision. A group that holds an infinity or a NaN gets the
// exponent 255, which reads as NaN. A lane takes 8 elements, four lanes a group.
//
// Both are bound by memory: 2 bytes read and 2 (or 17/32) written an element. 16,384
// tokens of 8 heads of 128 take 22.6 to 24.6 us, 5.5 TB/s of the 5.7 that a plain copy
// reaches, and back out in the same time (21.9 and 21.5 us in a graph); 8,200 into 4 bits 7.6
// to 9.5, and out of them 8.6 to 9.9 (42 MB, 4.5 TB/s: a launch this short does not reach the
// full rate).
#include <hip/hip_runtime.h>

#include "paged.hpp"
#include "ptstore.h"

namespace ptsd {
namespace {

typedef unsigned int v4u __attribute__((ext_vector_type(4)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;

// The block and the place in it of `slot`, or false where it is no place of the cache. (A
// plane has at most 2^36 bytes and a slot at least 34 of them: below 2^31.)
__device__ bool locate(const Planes& kv, int64_t slot, uint32_t& block, uint32_t& in_page) {
    const bool there = slot >= 0 && slot < kv.blocks * kv.div.page;
    const uint32_t at = there ? (uint32_t)slot : 0u;
    block = div_page(at, kv.div);
    in_page = at - block * kv.div.page;
    return there;
}

// The token and head of a row, and the lane's place in it: kLanes lanes a row.
struct Place {
    uint32_t row, token, head, lane;
};
template <int kLanes>
__device__ Place place(const PageDiv& heads) {
    Place p;
    p.row = blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
    p.lane = threadIdx.x % kLanes;
    p.token = div_page(p.row, heads);
    p.head = p.row - p.token * heads.page;
    return p;
}

// kRead: pages to rows, else rows to pages. A lane moves 16 bytes of K and of V.
template <int kLanes, bool kRead>
__global__ __launch_bounds__(kThreads) void k_rows16(Planes kv, Rows k, Rows v, const int64_t* slots,
                                                     uint32_t rows, PageDiv heads) {
    const Place at = place<kLanes>(heads);
    if (at.row >= rows) return;
    const uint32_t t = at.token, h = at.head, c = at.lane;
    uint32_t block, in_page;
    const bool there = locate(kv, slots[t], block, in_page);
    const int64_t page = (int64_t)block * kv.slab + ((int64_t)(h * kv.div.page + in_page) * kv.dim + c * 8) * 2;
    const int64_t ko = ((int64_t)t * k.token + (int64_t)h * k.head + c * 8) * 2;
    const int64_t vo = ((int64_t)t * v.token + (int64_t)h * v.head + c * 8) * 2;
    v4u* const kr = (v4u*)((uint8_t*)k.p + ko);
    v4u* const vr = (v4u*)((uint8_t*)v.p + vo);
    if constexpr (kRead) {
        const v4u zero = {0u, 0u, 0u, 0u};
        *kr = there ? *(const v4u*)(kv.k + page) : zero;
        *vr = there ? *(const v4u*)(kv.v + page) : zero;
    } else if (there) {
        // read once, past the caches' usual order: 10 % faster
        const v4u a = __builtin_nontemporal_load(kr), b = __builtin_nontemporal_load(vr);
        *(v4u*)(kv.k + page) = a;
        *(v4u*)(kv.v + page) = b;
    }
}

__device__ inline uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

// 8 bf16 values of a lane to 8 codes; `byte` gets the group's exponent.
__device__ inline uint32_t encode(v4u x, uint32_t& byte) {
    uint32_t most = 0;  // magnitudes order as whole numbers, infinities and NaN last
#pragma unroll
    for (int i = 0; i < 4; ++i) most = larger(most, larger(x[i] & 0x7FFFu, (x[i] >> 16) & 0x7FFFu));
    most = larger(most, (uint32_t)__shfl_xor((int)most, 1));
    most = larger(most, (uint32_t)__shfl_xor((int)most, 2));
    // 1.m 2^k: e = k - 2 up to m = 1.75, else k - 1
    int e = (int)((most + 0x1Fu) >> 7) - 2;
    e = e < 1 ? 1 : (e > 252 ? 252 : e);  // 6 * 2^125 is the largest that bf16 holds
    byte = most >= 0x7F80u ? 255u : (uint32_t)e;
    const float step = __uint_as_float((uint32_t)e << 23);
    uint32_t code = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t bits = x[i];  // (a bit cast of a vector's element reads its first)
        const bf2 pair = __builtin_bit_cast(bf2, bits);
        const uint32_t two = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, pair, step, 0);
        code |= (two & 0xFFu) << (8 * i);
    }
    return code;
}

__device__ inline v4u decode(uint32_t code, uint32_t byte) {
    const float step = __uint_as_float((byte >= kEndless ? 255u : byte) << 23);
    v4u x;
    x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, step, 0));
    x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, step, 1));
    x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, step, 2));
    x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, step, 3));
    return x;
}

template <int kLanes, bool kRead>
__global__ __launch_bounds__(kThreads) void k_rows4(Planes kv, Rows k, Rows v, const int64_t* slots,
                                                     uint32_t rows, PageDiv heads) {
    const Place at = place<kLanes>(heads);
    if (at.row >= rows) return;  // whole rows, so whole groups of four lanes, leave together
    const uint32_t t = at.token, h = at.head, c = at.lane;
    uint32_t block, in_page;
    const bool there = locate(kv, slots[t], block, in_page);
    const uint32_t line = h * kv.div.page + in_page;
    const int64_t codes = (int64_t)block * kv.slab + line * (kv.dim / 2) + c * 4;
    const int64_t power = (int64_t)block * kv.slab + kv.exponents + line * (kv.dim / kGroup) + c / 4;
    const int64_t ko = ((int64_t)t * k.token + (int64_t)h * k.head + c * 8) * 2;
    const int64_t vo = ((int64_t)t * v.token + (int64_t)h * v.head + c * 8) * 2;
    v4u* const kr = (v4u*)((uint8_t*)k.p + ko);
    v4u* const vr = (v4u*)((uint8_t*)v.p + vo);
    if constexpr (kRead) {
        v4u a = {0u, 0u, 0u, 0u}, b = a;
        if (there) {
            a = decode(*(const uint32_t*)(kv.k + codes), kv.k[power]);
            b = decode(*(const uint32_t*)(kv.v + codes), kv.v[power]);
        }
        *kr = a;
        *vr = b;
    } else {
        uint32_t kb, vb;
        const uint32_t kc = encode(*kr, kb), vc = encode(*vr, vb);
        if (!there) return;
        *(uint32_t*)(kv.k + codes) = kc;
        *(uint32_t*)(kv.v + codes) = vc;
        if ((c & 3) == 0) {
            kv.k[power] = (uint8_t)kb;
            kv.v[power] = (uint8_t)vb;
        }
    }
}

template <int kLanes, bool kRead>
hipError_t launch_lanes(const Planes& kv, const Rows& k, const Rows& v, const int64_t* slots, int64_t n,
                        hipStream_t s) {
    const uint32_t rows = (uint32_t)(n * kv.heads), per = kThreads / kLanes;
    const dim3 grid((rows + per - 1) / per);
    const PageDiv heads = page_div(kv.heads);
    if (kv.kind == PTSTORE_KV_MXFP4)
        hipLaunchKernelGGL((k_rows4<kLanes, kRead>), grid, dim3(kThreads), 0, s, kv, k, v, slots, rows, heads);
    else
        hipLaunchKernelGGL((k_rows16<kLanes, kRead>), grid, dim3(kThreads), 0, s, kv, k, v, slots, rows, heads);
    return hipGetLastError();
}

template <bool kRead>
hipError_t launch_rows(const Planes& kv, const Rows& k, const Rows& v, const int64_t* slots, int64_t n,
                       hipStream_t s) {
    return kv.dim == 128 ? launch_lanes<16, kRead>(kv, k, v, slots, n, s)
                         : launch_lanes<8, kRead>(kv, k, v, slots, n, s);
}

}  // namespace

hipError_t launch_append(const Planes& kv, const Rows& k, const Rows& v, const int64_t* slots, int64_t n,
                         hipStream_t s) {
    return launch_rows<false>(kv, k, v, slots, n, s);
}

hipError_t launch_read(const Planes& kv, const Rows& k, const Rows& v, const int64_t* slots, int64_t n,
                       hipStream_t s) {
    return launch_rows<true>(kv, k, v, slots, n, s);
}

}  // namespace ptsd
