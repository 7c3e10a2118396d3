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
// wants them (see attend.hpp), and V is read from LDS transposed. Two workgroups share a
// compute unit, so that one's exponentials run beside the other's products.
//
// 8 KV heads of 4 query heads, dim 128: a prompt of 8,192 tokens 582 to 650 us by the
// machine's clock under this load (1.9 to 2.0 GHz), 850 to 940 TFLOP/s; fp16 616 to 626, from
// 4-bit pages 530 to 615, values of zero 505: the same instructions at other power; dim 64
// 340 to 366. A large library product reaches 1,350; here the
// matrix units work in 43 % of the cycles, the vector units in about 40 % (a third of it
// exponentials), LDS in 35 %: two waves overlap little of the two.
#include <type_traits>

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
template <int D, bool kFour>
__device__ inline int turn_v(int row) {
    // the low bits are free, since a read takes all four columns: 4-bit rows, whose lanes
    // write columns 2 or 4 apart, turn by them too
    const int low = !kFour ? 0 : D == 128 ? row & 3 : (row >> 1) & 1;
    return (D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2) + low;
}

// A running maximum that is behind by up to this much (in powers of two) is kept:
// weights then reach 2^8 times the largest otherwise, and the output is rescaled a few
// times a row instead of at every new maximum. fp16 weights have the room for it; bf16 ones
// start that much lower, so that their sums stay in a float all the same.
constexpr float kBehind = 8.f;
template <bool kHalf>
constexpr float kRoom = Elem<kHalf>::kRoom + (kHalf ? 0.f : kBehind);

constexpr int kMostParts = 16;  // of a tile

// Floats of a part in the workspace: [4 dimensions][row], then rows' maxima and sums.
constexpr int part_floats(int dim) { return kPromptRows * (dim + 2); }

template <int D, bool kHalf, bool kFour>
__global__ __launch_bounds__(kThreads, 2) void k_prompt(AttendPlan p) {
    using E = Elem<kHalf>;
    using V8 = typename E::v8;
    constexpr int kSteps = D / 16;               // matrix steps over the dimension
    constexpr int kRow = D * 2;                  // bytes of a row in LDS
    constexpr int kLanes = kFour ? 4 : D / 8;    // lanes that load a row
    constexpr int kLoads = 16 * kLanes / 64;     // loads of a wave's 16 rows
    constexpr int kPieces = kFour ? D / 32 : 1;  // 16-byte pieces in LDS of a lane's load

    // two buffers of K, two of V
    constexpr int kTile = kKeys * kRow;
    __shared__ uint8_t s_mem[4 * kTile];
    __shared__ int s_endless;  // a V value that is not finite lies behind the first row's last key

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, half = lane >> 5;
    // (tile, KV head) `unit`, whole or part `part` of p.splits of its keys
    const int rest = (int)(blockIdx.x - p.whole);
    const int part = rest < 0 ? 0 : rest / p.rest, parts = rest < 0 ? 1 : p.splits;
    const int unit = rest < 0 ? (int)blockIdx.x : p.whole + rest % p.rest;
    const int head = unit % p.kv.heads;
    // the last tiles of a request see the most keys: they go first
    const Tile f = find_tile(p, (p.whole + p.rest) / p.kv.heads - 1 - unit / p.kv.heads, kPromptRows);
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
    const int all_steps = (end + kKeys - 1) / kKeys;
    const int step0 = (int)((int64_t)all_steps * part / parts);
    const int steps = (int)((int64_t)all_steps * (part + 1) / parts);  // this part's are [step0, steps)

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
    bool far = false;  // scores are scaled before the maximum is taken

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
    // LDS addresses of a lane, the rest of which are constants: the swizzles of a row do
    // not change with the parts of its number that are left out here. Writes: row
    // 16 wave + i rows of a load + .. (K: turned by i, too).
    const int at_row = 16 * wave + lane / kLanes;
    uint32_t k_write[kFour ? kPieces : kLoads], v_write[kFour ? kPieces : 1];
    if constexpr (kFour) {
#pragma unroll
        for (int c = 0; c < kPieces; ++c) {
            k_write[c] = at_row * kRow + ((((lane & 3) * kPieces + c) ^ turn_k<D>(at_row)) * 16);
            v_write[c] = at_row * kRow + ((((lane & 3) * kPieces + c) ^ turn_v<D, kFour>(at_row)) * 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            k_write[i] = at_row * kRow + (((lane % kLanes) ^ turn_k<D>(at_row + i * (64 / kLanes))) * 16);
        v_write[0] = at_row * kRow + (((lane % kLanes) ^ turn_v<D, kFour>(at_row)) * 16);
    }
    // K reads: row of K that accumulator row m of a 32-key piece stands for, so that lanes
    // then hold 8 consecutive keys of each 16; column 2 i + half.
    uint32_t k_read[kSteps];
    {
        const int m8 = n >> 3, row = 16 * (m8 >> 1) + 8 * ((n >> 2) & 1) + 4 * (m8 & 1) + (n & 3);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) k_read[i] = row * kRow + (((2 * i + half) ^ turn_k<D>(row)) * 16);
    }
    // V reads: 16 lanes take dimensions 16 (g & 1) .., keys 8 (g >> 1) .. of each 16.
    uint32_t v_read[D / 32];
    {
        const int g = lane >> 4, l16 = lane & 15, row = 8 * (g >> 1) + (l16 >> 2);
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
            v_read[i] = row * kRow + (((4 * i + 2 * (g & 1) + ((l16 & 3) >> 1)) ^ turn_v<D, kFour>(row)) * 16) + (l16 & 1) * 8;
    }

    // step t to LDS; V's rows that are not there as zeros (4-bit: as finite values)
    auto store = [&](auto buffer, uint64_t ok, int t) {
        constexpr int buf = decltype(buffer)::value;
        uint8_t* const km = s_mem + buf * kTile;
        uint8_t* const vm = s_mem + (2 + buf) * kTile;
        const bool edge = t * kKeys + kKeys - 1 > tile_sees;
        if (ok != ~0ull || edge) {
            bool endless = false;
            if constexpr (kFour) {
                vpow = keep_finite<D>(vpow, (ok >> lane) & 1, t * kKeys + lane > tile_sees, endless);
            } else {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int row = at_row + i * (64 / kLanes);
                    const bool in = (ok >> row) & 1;
                    if (!in) vreg[i] = v4u{0u, 0u, 0u, 0u};
                    if (in && t * kKeys + row > tile_sees) endless |= drop_endless<kHalf>(vreg[i]);
                }
            }
            if (endless) s_endless = 1;
        }
        if constexpr (kFour) {
            const int shift = (lane & 3) * (D / 4) / kGroup * 8;
            const float ks = step_of(((uint32_t)__shfl((int)kpow, at_row) >> shift) & 255u);
            const float vs = step_of(((uint32_t)__shfl((int)vpow, at_row) >> shift) & 255u);
#pragma unroll
            for (int c = 0; c < kPieces; ++c) {
                *(v4u*)(km + k_write[c]) = widen8(kreg[0][c], ks);
                *(v4u*)(vm + v_write[c]) = widen8(vreg[0][c], vs);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                *(v4u*)(km + k_write[i] + i * (64 / kLanes) * kRow) = kreg[i];
                *(v4u*)(vm + v_write[0] + i * (64 / kLanes) * kRow) = vreg[i];
            }
        }
    };

    if (threadIdx.x == 0) s_endless = 0;
    __syncthreads();
    int32_t entry = page_entry(p, table, step0 * kKeys + lane, end);
    uint64_t ok = 0, ok_next = 0;  // which keys of the step, and of the loaded one, are there
    bool there;
    if (step0 < steps) {
        const int32_t key = step0 * kKeys + lane;
        KeyRow place = key_row<D, kFour>(p.kv, entry, key, end, head_row, there);
        ok = __ballot(there);
        load(place);
        entry = page_entry(p, table, key + kKeys, end);
        store(std::integral_constant<int, 0>{}, ok, step0);
        if (step0 + 1 < steps) {
            place = key_row<D, kFour>(p.kv, entry, key + kKeys, end, head_row, there);
            ok_next = __ballot(there);
            load(place);
            entry = page_entry(p, table, key + 2 * kKeys, end);
        }
    }
    __syncthreads();

    auto turn = [&](auto buffer, int t) {
        constexpr int buf = decltype(buffer)::value;
        const uint8_t* const km = s_mem + buf * kTile;
        const uint8_t* const vm = s_mem + (2 + buf) * kTile;
        const int32_t at = t * kKeys;
        v16f s[2];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[c][e] = 0.f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int c = 0; c < 2; ++c)
                s[c] = E::mma32(__builtin_bit_cast(V8, *(const v4u*)(km + k_read[i] + c * 32 * kRow)), q[i], s[c]);
        if (t + 1 < steps) store(std::integral_constant<int, buf ^ 1>{}, ok_next, t + 1);
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
            seen = (seen & ok_now) >> (8 * half);
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
        auto scale_now = [&] {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[c][e] = product(s[c][e], p.scale2);
            most = product(most, p.scale2);
        };
        if (far) scale_now();
        float top2 = fmaxf(top, __builtin_fmaf(most, far ? 1.f : p.scale2, kRoom<kHalf>));
        // (far away, steps of the maximum can be 8 themselves: none is kept behind)
        if (__any(top2 > top + (far ? 0.f : kBehind))) {
            if (!far && __any(is_far(top2))) {
                far = true;
                scale_now();
                top2 = fmaxf(top, most + kRoom<kHalf>);
            }
            const float less = exp2_of(top - top2);
            sum *= less;
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[i][e] *= less;
            top = top2;
        }
        const float scale = far ? 1.f : p.scale2;
        v4u w[4];  // weights of 16 keys each
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[c][e] = exp2_of(__builtin_fmaf(s[c][e], scale, -top));
                sum += s[c][e];
            }
            // Weights enter the second product as 16-bit values, as V does; the sum takes them
            // as they are. Each is off by half a step of the type at most, as much as the
            // output's own rounding adds. Over many keys the errors average out; where one key has
            // nearly all the weight and the maximum is behind, they do not.
#pragma unroll
            for (int e = 0; e < 8; ++e)
                w[2 * c + (e >> 2)][e & 3] = pack2<kHalf>(s[c][2 * e], s[c][2 * e + 1]);
        }
        // column d of 16 keys, 8 of them a lane: two transposed reads
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            v4u vt[D / 32];
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                vt[i] = join(read_transposed(vm + v_read[i] + 16 * b * kRow),
                             read_transposed(vm + v_read[i] + (16 * b + 4) * kRow));
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                o[i] = E::mma32(__builtin_bit_cast(V8, vt[i]), __builtin_bit_cast(V8, w[b]), o[i]);
        }
        __syncthreads();
    };
    for (int t = step0; t < steps; t += 2) {
        turn(std::integral_constant<int, 0>{}, t);
        if (t + 1 < steps) turn(std::integral_constant<int, 1>{}, t + 1);
    }

    if (s_endless) {
        const int32_t from = tile_sees + 1 > step0 * kKeys ? tile_sees + 1 : step0 * kKeys;
        for (int32_t key = from; key < end && key < steps * kKeys; ++key) {
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
    if (parts > 1) {
        // four dimensions a lane, rows next to each other
        float* const to = p.parts + ((int64_t)(unit - p.whole) * parts + part) * part_floats(D);
        const int r = wave * 32 + n;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *(v4f*)(to + ((8 * i + 2 * a + half) * kPromptRows + r) * 4) =
                    v4f{o[i][4 * a], o[i][4 * a + 1], o[i][4 * a + 2], o[i][4 * a + 3]};
        if (half == 0) *(v2f*)(to + kPromptRows * D + 2 * r) = v2f{top, sum};
        return;
    }
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

// Joins the parts of tiles that have more than one: 32 rows of a (tile, KV head) a
// workgroup, a row and 8 dimensions a lane.
constexpr int kJoinRows = 32;

template <int D, bool kHalf>
__global__ __launch_bounds__(kJoinRows* D / 8) void k_prompt_join(AttendPlan p) {
    constexpr int kSlices = kPromptRows / kJoinRows;
    const int at = blockIdx.x / kSlices, unit = p.whole + at, head = unit % p.kv.heads;
    const Tile f = find_tile(p, (p.whole + p.rest) / p.kv.heads - 1 - unit / p.kv.heads, kPromptRows);
    if (f.tile < 0) return;
    const int r = blockIdx.x % kSlices * kJoinRows + threadIdx.x % kJoinRows, c = threadIdx.x / kJoinRows;
    const int row = f.tile * kPromptRows + r;
    if (row >= f.n * p.group) return;
    const float* const from = p.parts + (int64_t)at * p.splits * part_floats(D);
    float all = kLowest;
    for (int i = 0; i < p.splits; ++i)
        all = fmaxf(all, from[(int64_t)i * part_floats(D) + kPromptRows * D + 2 * r]);
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0}, total = 0.f;
#pragma unroll 4
    for (int i = 0; i < p.splits; ++i) {
        const float* part = from + (int64_t)i * part_floats(D);
        const v2f ms = *(const v2f*)(part + kPromptRows * D + 2 * r);
        const v4f a = *(const v4f*)(part + (2 * c * kPromptRows + r) * 4);
        const v4f b = *(const v4f*)(part + ((2 * c + 1) * kPromptRows + r) * 4);
        const float part_of = exp2_of(ms[0] - all);
        total += part_of * ms[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            acc[e] += part_of * a[e];
            acc[4 + e] += part_of * b[e];
        }
    }
    const float inv = total != 0.f ? 1.f / total : 0.f;
    const int token = row / p.group;
    const int64_t oh = (int64_t)head * p.group + (row - token * p.group);
    v4u x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = pack2<kHalf>(acc[2 * e] * inv, acc[2 * e + 1] * inv);
    *(v4u*)((uint8_t*)p.out.p + ((f.begin + token) * p.out.token + oh * p.out.head + c * 8) * 2) = x;
    if (p.lse && c == 0)
        p.lse[(f.begin + token) * p.q_heads + oh] =
            total != 0.f ? (all + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
}

template <int D, bool kHalf, bool kFour>
hipError_t run(const AttendPlan& p, hipStream_t s) {
    hipLaunchKernelGGL((k_prompt<D, kHalf, kFour>), dim3((unsigned)(p.whole + p.rest * p.splits)), dim3(kThreads), 0, s,
                       p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits < 2) return e;
    hipLaunchKernelGGL((k_prompt_join<D, kHalf>), dim3((unsigned)(p.rest * (kPromptRows / kJoinRows))),
                       dim3(kJoinRows * D / 8), 0, s, p);
    return hipGetLastError();
}

template <int D>
hipError_t run_kind(const AttendPlan& p, hipStream_t s) {
    if (p.kv.kind == PTSTORE_KV_MXFP4) return run<D, false, true>(p, s);
    return p.kv.kind == PTSTORE_KV_FP16 ? run<D, true, false>(p, s) : run<D, false, false>(p, s);
}

}  // namespace

// (tile, KV head) pairs of a last turn that are still split: 0.6 of the turn's places.
static int64_t most_rest(int cus) { return 2ll * cus * 3 / 5; }

// Two workgroups a compute unit run at once. Where a batch has fewer tiles than
// that, their keys are split so that all work; the tiles of a last turn that would be
// at most 0.6 full, likewise, up to four turns (past that, short tiles fill the
// end): with a second turn 0.55 full, 178 + 10 us so and 198 whole, 0.63 full, 150 + 10
// and 159. 2 requests of 128 tokens behind 4,000 (8 KV heads of 4) take 35 + 9 us split, 98
// whole. The host knows the number of tiles to within half a tile a request.
void split_prompt(AttendPlan* p, int cus) {
    const int64_t heads = p->kv.heads, slots = 2 * cus;
    const int64_t rows = p->n_tokens * p->group;
    const int64_t bound = p->R == 1 ? (rows + kPromptRows - 1) / kPromptRows
                                    : tile_bound(p->n_tokens, p->group, p->R, kPromptRows);
    const int64_t likely = p->R == 1 ? bound : (rows + (int64_t)p->R * (kPromptRows / 2)) / kPromptRows;
    int64_t rest = 0;  // tiles in parts, of each head
    if (bound * heads < slots)
        rest = bound;
    else if (likely * heads < 4 * slots)
        rest = likely * heads % slots / heads;
    int64_t splits = rest ? slots / (rest * heads) : 1;
    if (splits < 2 && rest < bound && rest * heads <= most_rest(cus)) splits = 2;
    // Ten steps a part at least, where the table is full: a prompt of 1,024 tokens takes
    // 26 + 8 us in two parts, 31 whole. The host knows the table's width and no request's
    // keys: in a table that is far wider than its requests short prompts get parts of a step,
    // or of none, and lose. Tight table, and one of 131,072 keys (in a graph, us):
    //
    //   tokens behind keys   64    256   1,024   4 x 256   8 x 200 / 800   64 / 1,000   512 / 4,000
    //   tight               8.2   12.5    31.0      14.2            45.0         30.5          65.0
    //   wide               24.4   27.4    36.2      19.1            48.8         26.5          60.8
    const int64_t most = (int64_t)p->max_blocks * p->kv.div.page / (10 * kKeys);
    if (splits > most) splits = most;
    if (splits < 2) rest = 0;
    p->whole = (int32_t)((bound - rest) * heads);
    p->rest = (int32_t)(rest * heads);
    p->splits = rest ? (int32_t)(splits < kMostParts ? splits : kMostParts) : 1;
}

int64_t prompt_workspace(const Planes& kv, int cus) {
    return 2ll * most_rest(cus) * part_floats(kv.dim) * (int64_t)sizeof(float);
}

hipError_t launch_prompt(const AttendPlan& p, hipStream_t s) {
    return p.kv.dim == 128 ? run_kind<128>(p, s) : run_kind<64>(p, s);
}

}  // namespace ptsd
