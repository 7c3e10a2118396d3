// Device parts that the attention kernels share (decode.hip, prompt.hip).
//
// Scores are computed transposed, S^T = K Q^T, and so is the output, O^T =
// V^T P^T: a query is a column of both, a lane holds one query's scores, and
// its share of P^T is in the registers where the second product wants it. The
// matrix instructions sum over 8 consecutive keys per lane; which key a row of
// K stands for is free, and is chosen (key_of_row) so that a lane's scores are
// those of 8 consecutive keys.
#pragma once

#include <hip/hip_runtime.h>

#include "paged.hpp"
#include "ptstore.h"

namespace ptsd {

typedef unsigned int v2u __attribute__((ext_vector_type(2)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));

// A 16-bit type's vectors and matrix instructions. The 4-bit cache is widened
// to bf16, which holds its values exactly.
template <bool kHalf>
struct Elem;

template <>
struct Elem<false> {
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    static constexpr uint32_t kExpMask = 0x7F807F80u;  // all ones: infinity or NaN
    // The largest weight is 2^-kRoom (prompt.hip: where a maximum is behind), so that sums of
    // 2^30 values near the type's largest, 2^128, stay in a float. Weights keep their bits: bf16
    // has a float's range.
    static constexpr float kRoom = 31.f;
    static __device__ v4f mma16(v8 a, v8 b, v4f c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ v16f mma32(v8 a, v8 b, v16f c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};

template <>
struct Elem<true> {
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    static constexpr uint32_t kExpMask = 0x7C007C00u;
    // The largest weight is 2^7, and 2^15 where a maximum may be behind (prompt.hip): the
    // type ends at 2^16, and its smallest value is then 2^-31 of the largest weight, so that
    // many keys of little weight each still count. No sum of its values leaves a float.
    static constexpr float kRoom = -7.f;
    static __device__ v4f mma16(v8 a, v8 b, v4f c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    static __device__ v16f mma32(v8 a, v8 b, v16f c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};

// Two floats to two 16-bit values, nearest even.
template <bool kHalf>
__device__ inline uint32_t pack2(float a, float b) {
    const v2f x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, typename Elem<kHalf>::v2));
}

// A weight of zero times an infinity would be a NaN. So in V's rows that some
// row of a tile must not see, values that are not finite are replaced by zeros
// before the product (true if there were any), and added at the end, by
// add_endless, to the rows that do see them.
template <bool kHalf>
__device__ inline bool drop_endless(v4u& x) {
    constexpr uint32_t lo = Elem<kHalf>::kExpMask & 0xFFFFu, hi = Elem<kHalf>::kExpMask & 0xFFFF0000u;
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool a = (x[i] & lo) == lo, b = (x[i] & hi) == hi;
        any |= a || b;
        x[i] &= (a ? 0u : 0xFFFFu) | (b ? 0u : 0xFFFF0000u);
    }
    return any;
}

// Four 16-bit rows' values of one column: lane i of 16 gives the address of 4
// values of row i / 4 and gets column i of the 4 x 16 piece.
__device__ inline v2u read_transposed(const uint8_t* lds) {
    typedef __attribute__((address_space(3))) v4s lds_v4s;
    return __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)lds));
}

__device__ inline v4u join(v2u a, v2u b) { return v4u{a[0], a[1], b[0], b[1]}; }

// The 32 codes of a lane's 16 bytes: piece `i` of four, 8 elements.
__device__ inline v4u widen8(uint32_t code, float step) {
    v4u x;
    x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, step, 0));
    x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, step, 1));
    x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, step, 2));
    x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, step, 3));
    return x;
}

// 2^(b - 127) of an exponent byte. From 253 on a code could leave bf16's range: all
// of them read as NaN, as 255 does.
__device__ inline float step_of(uint32_t byte) {
    return __uint_as_float((byte >= kEndless ? 255u : byte) << 23);
}

// Makes the wave wait for several exchanged values at once: one by one, as the
// compiler likes to place them, each costs a trip through LDS.
__device__ inline void together(uint32_t (&x)[1]) { asm volatile("" : "+v"(x[0])); }
__device__ inline void together(uint32_t (&x)[2]) { asm volatile("" : "+v"(x[0]), "+v"(x[1])); }
__device__ inline void together(uint32_t (&x)[4]) {
    asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));
}
__device__ inline void together(uint32_t (&x)[8]) {
    asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]),
                 "+v"(x[7]));
}

// Lowest score kept, a float's lowest number: what a row starts from instead of minus
// infinity, so that the differences of two such rows stay numbers.
constexpr float kLowest = -0x1.fffffep127f;

// A weight is 2^(score * scale - maximum), one fused operation whose product is exact, while
// the maximum is a rounded product. Where a float's steps are large, the difference of the
// two is no small number even for the largest score: at 2^31, up to 2^7, and its weight
// leaves the type. So from a maximum 2^20 away from zero on (a step is then 2^-3) a wave
// rounds the scaled scores first, each by itself, and a maximum is one of them.
constexpr float kFar = 0x1p20f;
__device__ inline bool is_far(float top) { return __builtin_fabsf(top) > kFar && top > kLowest; }

// A product that is rounded, whatever sum it enters.
__device__ inline float product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// A request's tile: its number among the request's tiles, and the request's
// numbers. `tile` < 0: no work.
struct Tile {
    int r, tile;
    int64_t begin;  // first token
    int32_t n;      // new tokens
    int64_t past;
};

// Finds tile number t of the batch. Every wave looks for itself, 64 requests at
// a time: request r's tiles start at offsets[r] * group / rows + r, which
// rises with r, so the lanes that start at or before t are counted.
__device__ inline Tile find_tile(const AttendPlan& p, int64_t t, int rows) {
    const int lane = threadIdx.x & 63;
    Tile f;
    f.tile = -1;
    int lo = 0, span = p.R;  // the request is in [lo, lo + span)
    while (span > 64) {
        const int step = (span + 63) / 64;
        const int r = lo + lane * step;
        const bool at = r < lo + span && p.offsets[r] * p.group / rows + r <= t;
        const int n = __popcll(__ballot(at));
        const int from = lo + (n > 0 ? n - 1 : 0) * step;
        span = lo + span - from < step ? lo + span - from : step;
        lo = from;
    }
    const int r = lo + lane;
    int64_t a = 0, b = 0;
    int32_t past = 0;
    const bool in = lane < span;
    if (in) {
        a = p.offsets[r];
        b = p.offsets[r + 1];
        past = p.context[r];
    }
    const int n = __popcll(__ballot(in && a * p.group / rows + r <= t));
    const int src = __builtin_amdgcn_readfirstlane(n > 0 ? n - 1 : 0);
    f.r = lo + src;
    const int64_t begin = ((int64_t)__builtin_amdgcn_readlane((int)(a >> 32), src) << 32) |
                          (uint32_t)__builtin_amdgcn_readlane((int)a, src);
    const int64_t end = ((int64_t)__builtin_amdgcn_readlane((int)(b >> 32), src) << 32) |
                        (uint32_t)__builtin_amdgcn_readlane((int)b, src);
    f.past = __builtin_amdgcn_readlane(past, src);
    if (begin < 0 || end < begin || end > p.n_tokens) return f;
    f.begin = begin;
    f.n = (int32_t)(end - begin);
    const int64_t tile = t - (begin * p.group / rows + f.r);
    if (tile < 0 || tile * rows >= (int64_t)f.n * p.group || (int64_t)f.n * p.group <= p.few_rows) return f;
    f.tile = (int)tile;
    return f;
}

// The block-table entry of key `key` of a request that has keys up to `end`. Past
// them it is the last one's (the first, if there is no key): loads need no branch, and
// key_row tells them apart.
__device__ inline int32_t page_entry(const AttendPlan& p, const int32_t* table, int32_t key, int32_t end) {
    const int32_t last = end > 0 ? end - 1 : 0;
    return table[div_page((uint32_t)(key < last ? key : last), p.kv.div)];
}

// A key's row of a head in a plane, in units of 16 bytes (a plane has at most 64 GiB),
// and the byte of its exponents in a 4-bit one. Block 0's first slot, and not `there`,
// if the key is at or past `end` or its page does not exist.
struct KeyRow {
    uint32_t at;
    uint64_t power;
};

template <int D, bool kFour>
__device__ inline KeyRow key_row(const Planes& kv, int32_t entry, int32_t key, int32_t end, uint32_t head_row,
                                 bool& there) {
    there = key < end && entry >= 0 && entry < (int32_t)kv.blocks;
    const uint32_t slot = (uint32_t)key - div_page((uint32_t)key, kv.div) * kv.div.page;
    const uint32_t block = there ? (uint32_t)entry : 0u, line = head_row + (there ? slot : 0u);
    KeyRow r;
    r.at = block * (kv.slab / 16) + line * (kFour ? D / 32 : D / 8);
    r.power = kFour ? (uint64_t)block * kv.slab + kv.exponents + line * (D / kGroup) : 0;
    return r;
}

// The exponents of a key's row: a byte each 32 dimensions.
template <int D>
__device__ inline uint32_t load_powers(const uint8_t* plane, uint64_t power) {
    if constexpr (D == 128)
        return *(const uint32_t*)(plane + power);
    else
        return *(const uint16_t*)(plane + power);
}

// Exponents with those of a key that is not there, or not finite behind `sees`, made
// smallest: its values are then finite, and a weight of zero keeps them out.
template <int D>
__device__ inline uint32_t keep_finite(uint32_t powers, bool there, bool behind, bool& endless) {
    if (!there) return 0;
    if (behind) {
#pragma unroll
        for (int i = 0; i < D; i += kGroup) {
            const uint32_t byte = (powers >> (i / kGroup * 8)) & 255u;
            if (byte >= kEndless) {
                powers &= ~(255u << (i / kGroup * 8));
                endless = true;
            }
        }
    }
    return powers;
}

// The value at dimension d of the V row `r`.
template <int D, bool kHalf, bool kFour>
__device__ inline float v_value(const Planes& kv, const KeyRow& r, int d) {
    const uint8_t* row = kv.v + ((uint64_t)r.at << 4);
    if constexpr (kFour) {
        const uint32_t code = row[d / 2] >> (4 * (d & 1));
        const uint32_t two = __builtin_bit_cast(
            uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, step_of(kv.v[r.power + d / kGroup]), 0));
        return __uint_as_float(two << 16);
    } else {
        const uint16_t x = *(const uint16_t*)(row + d * 2);
        return kHalf ? (float)__builtin_bit_cast(_Float16, x) : __uint_as_float((uint32_t)x << 16);
    }
}

// The largest of a column's values over the wave: of lanes 16 apart, or 32.
__device__ inline float larger_16_32(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float larger_32(float x) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Adds to a sum what drop_endless took from it.
__device__ inline float add_endless(float sum, float x) {
    return __builtin_isfinite(x) ? sum : sum + x;
}

}  // namespace ptsd
