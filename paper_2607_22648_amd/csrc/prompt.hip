// Attention of many query rows a KV head: whole prompts, and prompts behind a
// loaded prefix.
//
// Bound by the matrix units: 4 dim operations a (row, key) pair, and K and V
// come from L2 after the first tile of a request. A workgroup takes 128 rows
// ((token, head of the group) pairs of one KV head, so that its rows share K and V
// and the causal edge is 128 / group tokens wide), a wave 32 of them, and
// goes through the keys 64 at a time. K and V of a step pass through LDS once for
// all four waves, in two buffers: while a step is computed from one, the next
// is written to the other and the one after is on its way from memory to
// registers, which also widen 4-bit pages. One barrier a step.
//
// A wave computes S^T = K Q^T in 32 x 32 pieces, so that a lane holds 16 scores
// of one row, and the row's maximum and sum need one exchange between the wave's
// halves; the weights are then already where the second product O^T = V^T P^T
// wants them (see attend.hpp), and V is read from LDS transposed.
#include "attend.hpp"

namespace ptsd {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kKeys = 64;  // of a step

// Swizzles of rows in LDS: 16-byte column c of row r is at c ^ turn(r). K is read
// by 16 lanes of 16 consecutive rows, one column: all 16 have to differ. V is
// read by 32 lanes of 4 rows, 64 consecutive bytes each. A row of dim 64 is half
// of the banks, so that its lowest bit already separates two rows.
template <int D>
__device__ inline int turn_k(int row) {
    return D == 128 ? row & 15 : (row >> 1) & 7;
}
template <int D>
__device__ inline int turn_v(int row) {
    return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
}

// A running maximum that is behind by up to this much (in powers of two) is kept:
// weights then reach 2^8 instead of 1, which no type here minds, and the
// output is rescaled a few times a row instead of at every new maximum.
constexpr float kBehind = 8.f;

template <int D, bool kHalf, bool kFour>
__global__ __launch_bounds__(kThreads, 2) void k_prompt(AttendPlan p) {
    using E = Elem<kHalf>;
    using V8 = typename E::v8;
    constexpr int kSteps = D / 16;               // matrix steps over the dimension
    constexpr int kRow = D * 2;                  // bytes of a row in LDS
    constexpr int kLanes = kFour ? 4 : D / 8;    // lanes that load a row
    constexpr int kLoads = 16 * kLanes / 64;     // loads of a wave's 16 rows
    constexpr int kPieces = kFour ? D / 32 : 1;  // 16-byte pieces in LDS of a lane's load

    __shared__ uint8_t s_k[2][kKeys * kRow], s_v[2][kKeys * kRow];
    __shared__ int s_endless;  // a V value that is not finite lies behind the first row's last key

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int head = blockIdx.x % p.kv.heads;
    // the last tiles of a request see the most keys: they go first
    const int64_t tiles = gridDim.x / p.kv.heads;
    const Tile f = find_tile(p, tiles - 1 - blockIdx.x / p.kv.heads, kPromptRows);
    if (f.tile < 0) return;

    const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
    const int all_rows = f.n * p.group;
    const int row0 = f.tile * kPromptRows + wave * 32;
    const int row_at = row0 + n < all_rows ? row0 + n : all_rows - 1;
    const int token = row_at / p.group, sub = row_at - token * p.group;
    auto clip = [&](int64_t x) { return (int32_t)(x < -1 ? -1 : (x < limit ? x : limit - 1)); };
    // the last key that the tile's last and first row, the wave's first and this row see
    const int last_row = f.tile * kPromptRows + kPromptRows - 1 < all_rows ? f.tile * kPromptRows + kPromptRows - 1
                                                                            : all_rows - 1;
    const int32_t end = clip(f.past + last_row / p.group) + 1;
    const int first_row = row0 < all_rows ? row0 : all_rows - 1;
    const int32_t tile_sees = clip(f.past + f.tile * kPromptRows / p.group);
    const int32_t all_see = clip(f.past + first_row / p.group);
    const int32_t pos = clip(f.past + token);
    const int steps = (end + kKeys - 1) / kKeys;

    const int32_t* table = p.table + (int64_t)f.r * p.max_blocks;
    const uint32_t head_row = (uint32_t)head * p.kv.div.page;

    V8 q[kSteps];
    {
        const uint8_t* at = (const uint8_t*)p.q.p +
                            ((f.begin + token) * p.q.token + (int64_t)(head * p.group + sub) * p.q.head) * 2;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            q[s] = __builtin_bit_cast(V8, *(const v4u*)(at + (s * 16 + half * 8) * 2));
    }
    v16f o[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float top = kLowest, sum = 0.f;

    // a step's keys, one a lane; rows 16 wave .. + 15 are this wave's to load
    v4u kreg[kLoads], vreg[kLoads];
    uint32_t kpow = 0, vpow = 0;  // 4-bit: exponents of the lane's key
    const int lane_at = kFour ? (lane & 3) * (D / 8) : (lane % kLanes) * 16;
    auto load = [&](const KeyRow& r) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint64_t at =
                ((uint64_t)(uint32_t)__shfl((int)r.at, 16 * wave + i * (64 / kLanes) + lane / kLanes) << 4) + lane_at;
            if constexpr (kFour && D == 64) {
                const v2u a = *(const v2u*)(p.kv.k + at), b = *(const v2u*)(p.kv.v + at);
                kreg[i] = v4u{a[0], a[1], 0u, 0u};
                vreg[i] = v4u{b[0], b[1], 0u, 0u};
            } else {
                kreg[i] = *(const v4u*)(p.kv.k + at);
                vreg[i] = *(const v4u*)(p.kv.v + at);
            }
        }
        if constexpr (kFour) {
            kpow = load_powers<D>(p.kv.k, r.power);
            vpow = load_powers<D>(p.kv.v, r.power);
        }
    };
    // step t to LDS; V's rows that are not there as zeros (4-bit: as finite values)
    auto store = [&](int buf, uint64_t ok, int t, int here) {
        const bool edge = t * kKeys + kKeys - 1 > tile_sees;
        if (ok != ~0ull || edge) {
            bool endless = false;
            if constexpr (kFour) {
                vpow = keep_finite<D>(vpow, (ok >> lane) & 1, t * kKeys + lane > tile_sees, endless);
            } else {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int row = 16 * wave + i * (64 / kLanes) + lane / kLanes;
                    const bool in = (ok >> row) & 1;
                    if (!in) vreg[i] = v4u{0u, 0u, 0u, 0u};
                    if (in && t * kKeys + row > tile_sees) endless |= drop_endless<kHalf>(vreg[i]);
                }
            }
            if (endless) s_endless = 1;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = 16 * wave + i * (64 / kLanes) + here / kLanes;
            uint8_t* const kr = s_k[buf] + row * kRow;
            uint8_t* const vr = s_v[buf] + row * kRow;
            if constexpr (kFour) {
                const int shift = (here & 3) * (D / 4) / kGroup * 8;
                const float ks = step_of(((uint32_t)__shfl((int)kpow, row) >> shift) & 255u);
                const float vs = step_of(((uint32_t)__shfl((int)vpow, row) >> shift) & 255u);
                // turn_v leaves the low bits of the columns that 16 lanes write alike: rows
                // take a lane's words in orders of their own
                const bool one = D == 128 ? row & 1 : (row >> 1) & 1, two = D == 128 && (row & 2);
                const v4u a = one ? v4u{vreg[i][1], vreg[i][0], vreg[i][3], vreg[i][2]} : vreg[i];
                const v4u w = two ? v4u{a[2], a[3], a[0], a[1]} : a;
                const int turned = (one ? 1 : 0) | (two ? 2 : 0);
#pragma unroll
                for (int c = 0; c < kPieces; ++c) {
                    const int col = (here & 3) * kPieces + c, vcol = (here & 3) * kPieces + (c ^ turned);
                    *(v4u*)(kr + ((col ^ turn_k<D>(row)) * 16)) = widen8(kreg[i][c], ks);
                    *(v4u*)(vr + ((vcol ^ turn_v<D>(row)) * 16)) = widen8(w[c], vs);
                }
            } else {
                const int col = here % kLanes;
                *(v4u*)(kr + ((col ^ turn_k<D>(row)) * 16)) = kreg[i];
                *(v4u*)(vr + ((col ^ turn_v<D>(row)) * 16)) = vreg[i];
            }
        }
    };

    if (threadIdx.x == 0) s_endless = 0;
    __syncthreads();
    int32_t entry = steps > 0 ? page_entry(p, table, lane, end) : -1;
    uint64_t ok = 0, ok_next = 0;  // which keys of the step, and of the loaded one, are there
    bool there;
    if (steps > 0) {
        KeyRow place = key_row<D, kFour>(p.kv, entry, lane, end, head_row, there);
        ok = __ballot(there);
        load(place);
        entry = page_entry(p, table, kKeys + lane, end);
        store(0, ok, 0, lane);
        if (steps > 1) {
            place = key_row<D, kFour>(p.kv, entry, kKeys + lane, end, head_row, there);
            ok_next = __ballot(there);
            load(place);
            entry = page_entry(p, table, 2 * kKeys + lane, end);
        }
    }
    __syncthreads();

    for (int t = 0; t < steps; ++t) {
        const int buf = t & 1;
        const int32_t at = t * kKeys;
        // LDS addresses are formed anew each time: kept, they take registers of which
        // there are none to spare
        int here = lane;
        asm volatile("" : "+v"(here));
        v16f s[2];
        // row of K that accumulator row m of a 32-key piece stands for: lanes then hold
        // 8 consecutive keys of each 16
        const int m = here & 31, m8 = m >> 3;
        const int key_of_row = 16 * (m8 >> 1) + 8 * ((m >> 2) & 1) + 4 * (m8 & 1) + (m & 3);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int row = 32 * c + key_of_row;
            const uint8_t* kr = s_k[buf] + row * kRow;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[c][e] = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const v4u a = *(const v4u*)(kr + (((2 * i + (here >> 5)) ^ turn_k<D>(key_of_row)) * 16));
                s[c] = E::mma32(__builtin_bit_cast(V8, a), q[i], s[c]);
            }
        }
        if (t + 1 < steps) store(buf ^ 1, ok_next, t + 1, here);
        const uint64_t ok_now = ok;
        ok = ok_next;
        if (t + 2 < steps) {
            const int32_t key = (t + 2) * kKeys + lane;
            const KeyRow place = key_row<D, kFour>(p.kv, entry, key, end, head_row, there);
            ok_next = __ballot(there);
            load(place);
            entry = page_entry(p, table, key + kKeys, end);
        }
        // keys 32 c + 16 (e >> 3) + 8 half + (e & 7) in s[c][e]
        const bool some_hidden = ok_now != ~0ull || at + kKeys - 1 > all_see;
        if (some_hidden) {
            // the keys that are there and that the row sees, from bit 0 those of s[0][0] on
            const int32_t ahead = pos - at;
            uint64_t seen = ahead < 0 ? 0 : (ahead > 62 ? ~0ull : (2ull << ahead) - 1);
            seen = (seen & ok_now) >> (8 * (here >> 5));
            const uint32_t bits[2] = {(uint32_t)seen, (uint32_t)(seen >> 32)};
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!(bits[c] & (1u << (16 * (e >> 3) + (e & 7))))) s[c][e] = -INFINITY;
        }
        float most = -INFINITY;
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) most = fmaxf(most, s[c][e]);
        most = larger_32(most);
        const float top2 = fmaxf(top, most * p.scale2);
        if (__any(top2 > top + kBehind)) {
            const float less = exp2_of(top - top2);
            sum *= less;
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[i][e] *= less;
            top = top2;
        }
        v4u w[4];  // weights of 16 keys each
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[c][e] = exp2_of(__builtin_fmaf(s[c][e], p.scale2, -top));
                sum += s[c][e];
            }
            // weights enter the second product as 16-bit values, as V does: the error
            // of a weight is below the output's own rounding and averages over the keys
#pragma unroll
            for (int e = 0; e < 8; ++e)
                w[2 * c + (e >> 2)][e & 3] = pack2<kHalf>(s[c][2 * e], s[c][2 * e + 1]);
        }
        // column d of 16 keys, 8 of them a lane: two transposed reads
        const int g = here >> 4, l16 = here & 15;  // 16 lanes: dims 16 (g & 1), keys 8 (g >> 1)
        const int vrow0 = 8 * (g >> 1) + (l16 >> 2);
        const int vcol = 2 * (g & 1) + ((l16 & 3) >> 1), vin = (l16 & 1) * 8;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            v4u vt[D / 32];
            const int r0 = 16 * b + vrow0;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const int col = 4 * i + vcol;
                const v2u lo = read_transposed(s_v[buf] + r0 * kRow + ((col ^ turn_v<D>(vrow0)) * 16) + vin);
                const v2u hi =
                    read_transposed(s_v[buf] + (r0 + 4) * kRow + ((col ^ turn_v<D>(vrow0)) * 16) + vin);
                vt[i] = join(lo, hi);
            }
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                o[i] = E::mma32(__builtin_bit_cast(V8, vt[i]), __builtin_bit_cast(V8, w[b]), o[i]);
        }
        __syncthreads();
    }

    if (s_endless) {
        for (int32_t key = tile_sees + 1; key < end; ++key) {
            const KeyRow row =
                key_row<D, kFour>(p.kv, page_entry(p, table, key, end), key, end, head_row, there);
            if (!there || key > pos) continue;
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    o[i][e] = add_endless(
                        o[i][e], v_value<D, kHalf, kFour>(p.kv, row, 32 * i + 8 * (e >> 2) + 4 * half + (e & 3)));
        }
    }
    if (row0 + n >= all_rows) return;  // both halves of a row leave together
    sum += __shfl_xor(sum, 32);
    // no key, or none with a weight: zeros, and the logarithm of nothing
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    const int64_t oh = (int64_t)head * p.group + sub;
    uint8_t* const to = (uint8_t*)p.out.p + ((f.begin + token) * p.out.token + oh * p.out.head) * 2;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int a = 0; a < 4; a += 2) {
            // 4 dimensions here, the next 4 in the other half: trade, and write 8 a lane
            v4u x;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t even = pack2<kHalf>(o[i][4 * a + 2 * h] * inv, o[i][4 * a + 2 * h + 1] * inv);
                const uint32_t odd = pack2<kHalf>(o[i][4 * a + 4 + 2 * h] * inv, o[i][4 * a + 4 + 2 * h + 1] * inv);
                const auto both = __builtin_amdgcn_permlane32_swap(even, odd, false, false);
                x[h] = both[0];
                x[2 + h] = both[1];
            }
            *(v4u*)(to + (32 * i + 8 * (a + half)) * 2) = x;
        }
    if (p.lse && half == 0)
        p.lse[(f.begin + token) * p.q_heads + oh] =
            sum != 0.f ? (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f : -INFINITY;
}

template <int D, bool kHalf, bool kFour>
hipError_t run(const AttendPlan& p, hipStream_t s) {
    const int64_t units = tile_bound(p.n_tokens, p.group, p.R, kPromptRows) * p.kv.heads;
    hipLaunchKernelGGL((k_prompt<D, kHalf, kFour>), dim3((unsigned)units), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

template <int D>
hipError_t run_kind(const AttendPlan& p, hipStream_t s) {
    if (p.kv.kind == PTSTORE_KV_MXFP4) return run<D, false, true>(p, s);
    return p.kv.kind == PTSTORE_KV_FP16 ? run<D, true, false>(p, s) : run<D, false, false>(p, s);
}

}  // namespace

hipError_t launch_prompt(const AttendPlan& p, hipStream_t s) {
    return p.kv.dim == 128 ? run_kind<128>(p, s) : run_kind<64>(p, s);
}

}  // namespace ptsd
