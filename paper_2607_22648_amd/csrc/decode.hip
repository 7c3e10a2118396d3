// Attention of few query rows a KV head: single tokens, and the few of a draft
// that is checked.
//
// Bound by memory: a request's K and V are read once and every other byte is
// small beside them. So a request's keys are split into parts, one workgroup
// each (flash-decoding in form: each part keeps its own maximum and sum, and a
// second kernel joins them), and what matters is bytes in flight.
//
// A workgroup is four waves that share nothing until the end: wave w takes
// every fourth step of keys of the part. A step's K goes from memory straight into
// the matrix instruction's operand registers (16 keys a row group, 64
// consecutive bytes of a row by four lanes), its V through 8 KiB of LDS that only
// this wave uses, written as rows and read transposed. The next step's loads
// are issued as soon as a register is free, so that each wave keeps a step's
// bytes in flight while it computes.
//
// Query rows are the (token, head of the group) pairs of one KV head, 16 to a
// tile: with 4 heads to a KV head a single token fills 4 of the 16 columns, and
// the matrix instructions idle for the rest, which costs nothing here.
#include "attend.hpp"

namespace ptsd {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;

// Floats of one (tile, KV head, part) in the workspace: rows, maxima, sums.
constexpr int part_floats(int dim) { return kDecodeRows * (dim + 2); }

// K and V are read once: past the caches' usual order, so that they leave the
// parts' results there.
__device__ inline v4u once16(const uint8_t* p) { return __builtin_nontemporal_load((const v4u*)p); }
__device__ inline v2u once8(const uint8_t* p) { return __builtin_nontemporal_load((const v2u*)p); }

// Swizzle of K's rows in LDS: 16-byte column c of row r is at c ^ turn(r). 16 lanes
// read one column of rows {0-3, 8-11, 16-19, 24-27} (or those 4 further on).
template <int D>
__device__ inline int turn_k(int row) {
    return D == 128 ? (row & 3) | ((row >> 3) & 3) << 2 : ((row >> 1) & 1) | ((row >> 3) & 3) << 1;
}

// And of V's: two groups of 16 lanes read rows {0-3} and {8-11} (or {16-19} and {24-27}), 32
// bytes each, in one pass of the banks: eight rows have to differ in the upper
// bits. Rows of 128 bytes (dim 64) already differ by parity.
template <int D>
__device__ inline int turn_v(int row) {
    if constexpr (D == 128)
        return 2 * ((row & 3) + 4 * ((row >> 3) & 1));
    else
        return 2 * (((row >> 1) & 1) + 2 * ((row >> 3) & 1));
}

template <int D, bool kHalf, bool kFour>
__global__ __launch_bounds__(kThreads, 2) void k_decode(AttendPlan p) {
    using E = Elem<kHalf>;
    constexpr int kKeys = kFour ? 64 : 32;        // keys of a step
    constexpr int kGroups = kKeys / 16;           // row groups of 16 keys
    constexpr int kSteps = D / 32;                // matrix steps over the dimension
    constexpr int kRow = D * 2;                   // bytes of a row of V in LDS
    constexpr int kLanes = D / 8;                 // lanes that move a 16-bit row
    constexpr int kPieces = 32 * kLanes / 64;     // loads of 32 rows by a wave
    constexpr int kOut = D + 4;                   // floats of an output row in LDS, padded
    // 4-bit: a lane takes a quarter of a row of K, D / 8 bytes; four lanes of V
    constexpr int kWords = D / 32;                // 32-bit words of that
    constexpr int kVKeys = 64 / 4;                // rows of V a load covers

    __shared__ union {
        uint8_t v[kWaves][32 * kRow];
        float o[kWaves][kDecodeRows * kOut];
    } s_mem;
    __shared__ float s_max[kWaves][kDecodeRows], s_sum[kWaves][kDecodeRows];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = lane & 15, h4 = lane >> 4;  // query column, quarter
    const int part = blockIdx.x % p.splits;
    const int64_t unit = blockIdx.x / p.splits;  // tile, KV head
    const int head = (int)(unit % p.kv.heads);
    const Tile f = find_tile(p, unit / p.kv.heads, kDecodeRows);
    if (f.tile < 0) return;

    // the tile's rows see keys up to `last`; those of this part are [k0, k1)
    const int rows_left = f.n * p.group - f.tile * kDecodeRows;
    const int rows = rows_left < kDecodeRows ? rows_left : kDecodeRows;
    const int row = f.tile * kDecodeRows + (n < rows ? n : rows - 1);
    const int token = row / p.group, sub = row - token * p.group;
    const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
    const int64_t last = f.past + (f.tile * kDecodeRows + rows - 1) / p.group;
    int64_t seen = last + 1;
    seen = seen < 0 ? 0 : (seen > limit ? limit : seen);
    const int32_t end = (int32_t)seen;
    const int32_t k0 = part * p.part_keys;
    if (k0 >= end && part > 0) return;
    const int32_t k1 = end - k0 < p.part_keys ? end : k0 + p.part_keys;
    const int64_t pos64 = f.past + token;  // the last key this lane's query sees
    const int32_t pos = pos64 < limit ? (int32_t)pos64 : (int32_t)limit;
    const int64_t first64 = f.past + f.tile * kDecodeRows / p.group;
    const int32_t all_see = first64 < limit ? (int32_t)first64 : (int32_t)limit;

    const int32_t* table = p.table + (int64_t)f.r * p.max_blocks;
    const uint32_t head_row = (uint32_t)head * p.kv.div.page;

    // queries: column n, 8 consecutive dimensions a lane (4-bit: those of its quarter of a row)
    v4u q[kSteps];
    {
        const uint8_t* at = (const uint8_t*)p.q.p +
                            ((f.begin + token) * p.q.token + (int64_t)(head * p.group + sub) * p.q.head) * 2;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            q[s] = *(const v4u*)(at + (kFour ? h4 * (D / 4) + s * 8 : s * 32 + h4 * 8) * 2);
    }

    v4f o[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i] = v4f{0, 0, 0, 0};
    float top = kLowest, sum = 0.f;

    // K row of this lane within a row group: key_of_row
    const int key_of_row = 8 * (n >> 2) + (n & 3);
    // the step's keys, one a lane (32 keys: the upper half repeats them)
    const int step_key = lane & (kKeys - 1);
    const int32_t stride = kKeys * kWaves;

    v4u kreg[kFour ? kGroups : kPieces], vreg[kFour ? kKeys / kVKeys : kPieces];
    uint32_t kpow = 0, vpow = 0;  // 4-bit: exponents of the lane's key

    // A lane's bytes of the rows that the lanes hold: the places in a plane go round
    // the wave in 32 bits.
    const uint8_t* const kbase = p.kv.k + (kFour ? h4 * (D / 8) : (lane % kLanes) * 16);
    const uint8_t* const vbase = p.kv.v + (kFour ? (lane & 3) * (D / 8) : (lane % kLanes) * 16);
    auto row_at = [&](const uint8_t* base, const KeyRow& r, int key) {
        return base + ((uint64_t)(uint32_t)__shfl((int)r.at, key) << 4);
    };
    auto four = [&](const uint8_t* at) {
        if constexpr (D == 128) return once16(at);
        const v2u x = once8(at);
        return v4u{x[0], x[1], 0u, 0u};
    };
    auto load_k = [&](const KeyRow& r) {
        if constexpr (kFour) {
            kpow = load_powers<D>(p.kv.k, r.power);
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
                kreg[g] = four(row_at(kbase, r, 32 * (g >> 1) + 4 * (g & 1) + key_of_row));
        } else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) kreg[i] = once16(row_at(kbase, r, i * (64 / kLanes) + lane / kLanes));
        }
    };
    auto load_v = [&](const KeyRow& r) {
        if constexpr (kFour) {
            vpow = load_powers<D>(p.kv.v, r.power);
#pragma unroll
            for (int i = 0; i < kKeys / kVKeys; ++i) vreg[i] = four(row_at(vbase, r, i * kVKeys + (lane >> 2)));
        } else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) vreg[i] = once16(row_at(vbase, r, i * (64 / kLanes) + lane / kLanes));
        }
    };
    // the exponent of the lane's quarter q of row `key`
    auto power = [&](uint32_t pow, int key, int quarter) {
        return ((uint32_t)__shfl((int)pow, key) >> (quarter * (D / 4) / kGroup * 8)) & 255u;
    };

    // The order of loads is fixed (a wait for one waits for all before it): the page
    // entries of the step after next, the next step's K, the next step's V. Past the
    // part's end they read block 0, which costs less than a branch.
    int32_t at = k0 + wave * kKeys;
    bool there = false;
    KeyRow place;
    uint64_t valid = 0;
    int32_t entry = -1;
    if (at < k1) {
        entry = page_entry(p, table, at + step_key, k1);
        place = key_row<D, kFour>(p.kv, entry, at + step_key, k1, head_row, there);
        valid = __ballot(there);
        entry = page_entry(p, table, at + stride + step_key, k1);
        __builtin_amdgcn_sched_barrier(0);
        load_k(place);
        __builtin_amdgcn_sched_barrier(0);
        load_v(place);
        __builtin_amdgcn_sched_barrier(0);
    }
    uint8_t* const lds = s_mem.v[wave];
    bool endless = false;  // a V value that is not finite lies behind the first row's last key

    while (at < k1) {
        // scores of column n: keys 32 b + 8 h4 + 4 (g & 1) + i in s[g][i], b = g >> 1
        v4f s[kGroups];
        if constexpr (!kFour) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int key = i * (64 / kLanes) + lane / kLanes;
                *(v4u*)(lds + key * kRow + (((lane % kLanes) ^ turn_k<D>(key)) * 16)) = kreg[i];
            }
            __builtin_amdgcn_wave_barrier();
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            s[g] = v4f{0, 0, 0, 0};
            const int key = 4 * (g & 1) + key_of_row;
            const float step = kFour ? step_of(power(kpow, 32 * (g >> 1) + key, h4)) : 0.f;
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                v4u a;
                if constexpr (kFour)
                    a = widen8(kreg[g][t], step);
                else
                    a = *(const v4u*)(lds + key * kRow + (((4 * t + h4) ^ turn_k<D>(key)) * 16));
                s[g] = E::mma16(__builtin_bit_cast(typename E::v8, a), __builtin_bit_cast(typename E::v8, q[t]),
                                s[g]);
            }
        }
        __builtin_amdgcn_wave_barrier();
        const int32_t next = at + stride;
        const uint64_t ok = valid;
        place = key_row<D, kFour>(p.kv, entry, next + step_key, k1, head_row, there);
        valid = __ballot(there);
        entry = page_entry(p, table, next + stride + step_key, k1);
        __builtin_amdgcn_sched_barrier(0);
        load_k(place);
        __builtin_amdgcn_sched_barrier(0);

        constexpr uint64_t kAll = kKeys == 64 ? ~0ull : 0xFFFFFFFFull;
        const bool edge = k1 - 1 > all_see && at + kKeys - 1 > all_see;
        const bool some_hidden = (ok & kAll) != kAll || edge;
        if (some_hidden) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int key = 32 * (g >> 1) + 8 * h4 + 4 * (g & 1);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!((ok >> (key + i)) & 1) || at + key + i > pos) s[g][i] = -INFINITY;
            }
            // V's rows that are not there become zeros (4-bit: finite)
            if constexpr (kFour) {
                vpow = keep_finite<D>(vpow, (ok >> lane) & 1, at + lane > all_see, endless);
            } else {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int key = i * (64 / kLanes) + lane / kLanes;
                    const bool in = (ok >> key) & 1;
                    if (!in) vreg[i] = v4u{0u, 0u, 0u, 0u};
                    if (in && at + key > all_see) endless |= drop_endless<kHalf>(vreg[i]);
                }
            }
        }
        float most = -INFINITY;
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = fmaxf(most, s[g][i]);
        most = larger_16_32(most);
        const float top2 = fmaxf(top, most * p.scale2);
        if (__any(top2 > top)) {
            const float less = exp2_of(top - top2);
            sum *= less;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[i] *= less;
            top = top2;
        }
        v4u w[kKeys / 32];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[g][i] = exp2_of(__builtin_fmaf(s[g][i], p.scale2, -top));
                sum += s[g][i];
            }
            // weights enter the second product as 16-bit values, as V does: the error
            // of a weight is below the output's own rounding and averages over the keys
            w[g >> 1][2 * (g & 1)] = pack2<kHalf>(s[g][0], s[g][1]);
            w[g >> 1][2 * (g & 1) + 1] = pack2<kHalf>(s[g][2], s[g][3]);
        }

#pragma unroll
        for (int b = 0; b < kKeys / 32; ++b) {
            // V's rows of 32 keys into LDS
            if constexpr (kFour) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int key = i * kVKeys + (lane >> 2), j = 2 * b + i;
                    const float step = step_of(power(vpow, 32 * b + key, lane & 3));
#pragma unroll
                    for (int c = 0; c < kWords; ++c) {
                        const int col = (lane & 3) * kWords + c;
                        *(v4u*)(lds + key * kRow + ((col ^ turn_v<D>(key)) * 16)) = widen8(vreg[j][c], step);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int key = i * (64 / kLanes) + lane / kLanes;
                    *(v4u*)(lds + key * kRow + (((lane % kLanes) ^ turn_v<D>(key)) * 16)) = vreg[i];
                }
            }
            __builtin_amdgcn_wave_barrier();
            if (b == kKeys / 32 - 1) {
                __builtin_amdgcn_sched_barrier(0);
                load_v(place);
                __builtin_amdgcn_sched_barrier(0);
            }
            // column d of 32 keys, 8 of them a lane: two transposed reads
            const int vrow = 8 * h4 + (n >> 2);
            v4u vt[D / 16];
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const int col = 2 * i + ((n & 3) >> 1), in = (n & 1) * 8;
                const v2u lo = read_transposed(lds + vrow * kRow + ((col ^ turn_v<D>(vrow)) * 16) + in);
                const v2u hi = read_transposed(lds + (vrow + 4) * kRow + ((col ^ turn_v<D>(vrow + 4)) * 16) + in);
                vt[i] = join(lo, hi);
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                o[i] = E::mma16(__builtin_bit_cast(typename E::v8, vt[i]),
                                __builtin_bit_cast(typename E::v8, w[b]), o[i]);
            __builtin_amdgcn_wave_barrier();
        }
        at = next;
    }
    if (__any(endless)) {
        for (int32_t first = k0 + wave * kKeys; first < k1; first += stride)
            for (int32_t key = first; key < k1 && key < first + kKeys; ++key) {
                const KeyRow row = key_row<D, kFour>(p.kv, page_entry(p, table, key, k1), key, k1, head_row, there);
                if (!there || key <= all_see || key > pos) continue;
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[i][e] = add_endless(o[i][e], v_value<D, kHalf, kFour>(p.kv, row, 16 * i + 4 * h4 + e));
            }
    }

    // join the four waves; then this part's rows go out, or to the workspace
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    __syncthreads();  // every wave is done with its V
    if (h4 == 0) {
        s_max[wave][n] = top;
        s_sum[wave][n] = sum;
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) *(v4f*)&s_mem.o[wave][n * kOut + 16 * i + 4 * h4] = o[i];
    __syncthreads();
    constexpr int kRowLanes = D / 8;
    const int orow = threadIdx.x / kRowLanes, oc = threadIdx.x % kRowLanes;
    if (orow >= rows) return;
    float all = kLowest;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all = fmaxf(all, s_max[w][orow]);
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0}, total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float part_of = exp2_of(s_max[w][orow] - all);
        total += part_of * s_sum[w][orow];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += part_of * s_mem.o[w][orow * kOut + oc * 8 + e];
    }
    if (end > p.part_keys) {
        float* to = p.parts + ((uint64_t)unit * p.splits + part) * part_floats(D);
        *(v4f*)(to + orow * D + oc * 8) = v4f{acc[0], acc[1], acc[2], acc[3]};
        *(v4f*)(to + orow * D + oc * 8 + 4) = v4f{acc[4], acc[5], acc[6], acc[7]};
        if (oc == 0) {
            to[kDecodeRows * D + orow] = all;
            to[kDecodeRows * (D + 1) + orow] = total;
        }
        return;
    }
    const int out_row = f.tile * kDecodeRows + orow;
    const int ot = out_row / p.group, os = out_row - ot * p.group;
    const int64_t oh = (int64_t)head * p.group + os;
    // no key, or none with a weight: zeros, and the logarithm of nothing
    const float inv = total != 0.f ? 1.f / total : 0.f;
    v4u x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = pack2<kHalf>(acc[2 * e] * inv, acc[2 * e + 1] * inv);
    *(v4u*)((uint8_t*)p.out.p + ((f.begin + ot) * p.out.token + oh * p.out.head + oc * 8) * 2) = x;
    if (p.lse && oc == 0)
        p.lse[(f.begin + ot) * p.q_heads + oh] =
            total != 0.f ? (all + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
}

// Joins the parts of tiles that have more than one: a workgroup a (tile, KV head).
template <int D, bool kHalf>
__global__ __launch_bounds__(kThreads) void k_join(AttendPlan p) {
    const int64_t unit = blockIdx.x;
    const int head = (int)(unit % p.kv.heads);
    const Tile f = find_tile(p, unit / p.kv.heads, kDecodeRows);
    if (f.tile < 0) return;
    const int rows_left = f.n * p.group - f.tile * kDecodeRows;
    const int rows = rows_left < kDecodeRows ? rows_left : kDecodeRows;
    const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
    int64_t seen = f.past + (f.tile * kDecodeRows + rows - 1) / p.group + 1;
    if (seen > limit) seen = limit;
    if (seen <= p.part_keys) return;
    const int parts = (int)((seen + p.part_keys - 1) / p.part_keys);
    constexpr int kRowLanes = D / 8;
    const int orow = threadIdx.x / kRowLanes, oc = threadIdx.x % kRowLanes;
    if (orow >= rows) return;
    const float* from = p.parts + (uint64_t)unit * p.splits * part_floats(D);
    float all = kLowest;
    for (int i = 0; i < parts; ++i)
        all = fmaxf(all, from[(int64_t)i * part_floats(D) + kDecodeRows * D + orow]);
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0}, total = 0.f;
    for (int i = 0; i < parts; ++i) {
        const float* part = from + (int64_t)i * part_floats(D);
        const float part_of = exp2_of(part[kDecodeRows * D + orow] - all);
        total += part_of * part[kDecodeRows * (D + 1) + orow];
        const v4f a = *(const v4f*)(part + orow * D + oc * 8), b = *(const v4f*)(part + orow * D + oc * 8 + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            acc[e] += part_of * a[e];
            acc[4 + e] += part_of * b[e];
        }
    }
    const int out_row = f.tile * kDecodeRows + orow;
    const int ot = out_row / p.group, os = out_row - ot * p.group;
    const int64_t oh = (int64_t)head * p.group + os;
    const float inv = total != 0.f ? 1.f / total : 0.f;
    v4u x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = pack2<kHalf>(acc[2 * e] * inv, acc[2 * e + 1] * inv);
    *(v4u*)((uint8_t*)p.out.p + ((f.begin + ot) * p.out.token + oh * p.out.head + oc * 8) * 2) = x;
    if (p.lse && oc == 0)
        p.lse[(f.begin + ot) * p.q_heads + oh] =
            total != 0.f ? (all + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
}

template <int D, bool kHalf, bool kFour>
hipError_t run(const AttendPlan& p, hipStream_t s) {
    const int64_t units = tile_bound(p.n_tokens, p.group, p.R, kDecodeRows) * p.kv.heads;
    hipLaunchKernelGGL((k_decode<D, kHalf, kFour>), dim3((unsigned)(units * p.splits)), dim3(kThreads), 0, s, p);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1) {
        hipLaunchKernelGGL((k_join<D, kHalf>), dim3((unsigned)units), dim3(kThreads), 0, s, p);
        e = hipGetLastError();
    }
    return e;
}

template <int D>
hipError_t run_kind(const AttendPlan& p, hipStream_t s) {
    if (p.kv.kind == PTSTORE_KV_MXFP4) return run<D, false, true>(p, s);
    return p.kv.kind == PTSTORE_KV_FP16 ? run<D, true, false>(p, s) : run<D, false, false>(p, s);
}

}  // namespace

hipError_t launch_decode(const AttendPlan& p, hipStream_t s) {
    return p.kv.dim == 128 ? run_kind<128>(p, s) : run_kind<64>(p, s);
}

}  // namespace ptsd
