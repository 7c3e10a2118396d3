// Attention of prompts over a latent cache in the expanded form: keys and values of every head are formed
// from the rows first, and attention over them takes fewer operations a (row, key) than in the latent space.
//
// A formed value lies between the 16-bit ones that products take. Rounded to one of them it would
// make scores, and the logarithms of their sums, as coarse; so it is kept as two, the nearest and what
// is left, 2^-16 (2^-22) of it off. Scores take 2 (128 + 128 + 64) operations a (row, key), the outputs
// 2 (128 + 128), where the latent space has 2 (576 + 512).
//
// Forming them is a matrix product: 128 keys and all of their latent values stay in LDS while a workgroup goes
// through the matrices of several heads, two at a time, which its waves read from L2 into registers, 64 of a
// head's 256 rows each. What comes out is packed by head.
//
// The attention is that of prompt.hip: 128 tokens of a head a workgroup, 32 a wave, S^T = K Q^T and
// O^T = V^T P^T. Keys lie next to each other and need no conversion, so they go to LDS without passing
// registers, 32 a step, into one of two buffers while the other is computed from. Two workgroups share a
// compute unit.
//
// Measured: 6 prompts of 33 to 3,500 tokens, 16 heads, 79 us for forming 10,599 keys (44 GFLOP) and 290 for the
// attention (matrix units 46 % of the cycles, other vector instructions 28; with 1.6 waves a SIMD they add up); 4 requests
// behind up to 3,584 tokens, 32 heads, 168 (12,828 keys; 420 MB written) and 246.
#include <type_traits>

#include "attend.hpp"
#include "latent.hpp"
#include "lds_fetch.hpp"

namespace ptsd {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kFormKeys = 128;  // of a workgroup that forms keys and values
constexpr int kFormWaves = 8, kFormThreads = kFormWaves * 64;  // four for a head
constexpr int kFewKeys = 32;    // of a workgroup where there are few keys
constexpr int kFewTurns = 4;    // workgroups of few keys a compute unit, at most
constexpr int kGroupTurns = 1;  // workgroups of eight waves of the attention a compute unit, at most
constexpr int kDies = 8;
constexpr int kDieBytes = 2 << 20;  // of matrices that a die goes through: half of its L2
constexpr int kKeys = 32;       // of a step of the attention
constexpr int kRow = 512;       // bytes of a formed key, or value: 128 nearest values, 128 of what is left

// The packed key x: its request (the last that begins at or before it), and its row's place in units of 16 bytes.
__device__ inline bool row_of(const ExpandedPlan& p, int64_t x, uint32_t& at) {
    int lo = 0, span = p.R;
    while (span > 1) {
        const int half = span / 2;
        const bool up = p.key_offsets[lo + half] <= x;
        lo = up ? lo + half : lo;
        span = up ? span - half : half;
    }
    at = 0;
    if (x >= p.n_keys || p.R < 1) return false;
    const int64_t first = p.key_offsets[lo];
    if (first < 0 || first > x || x >= p.key_offsets[lo + 1]) return false;
    const int64_t key = x - first;
    if (key >= (int64_t)p.max_blocks * p.kv.div.page) return false;
    const uint32_t column = div_page((uint32_t)key, p.kv.div);
    const int32_t entry = p.table[(int64_t)lo * p.max_blocks + column];
    if (entry < 0 || entry >= p.kv.blocks) return false;
    at = ((uint32_t)entry * p.kv.div.page + ((uint32_t)key - column * p.kv.div.page)) * p.kv.line;
    return true;
}

// Two floats to their nearest 16-bit values, and what is left of them to two more (nothing of one that is not
// finite, or becomes so).
template <bool kHalf>
__device__ inline uint32_t split2(float a, float b, uint32_t& left) {
    const uint32_t near = pack2<kHalf>(a, b);
    const typename Elem<kHalf>::v2 two = __builtin_bit_cast(typename Elem<kHalf>::v2, near);
    const float x = a - (float)two[0], y = b - (float)two[1];
    left = pack2<kHalf>(__builtin_isfinite(x) ? x : 0.f, __builtin_isfinite(y) ? y : 0.f);
    return near;
}

template <int L, bool kHalf>
__global__ __launch_bounds__(kFormThreads) void k_form(ExpandedPlan p) {
    using E = Elem<kHalf>;
    using V8 = typename E::v8;
    constexpr int kLine = L * 2 + 16;  // bytes in LDS: 16 lanes that read one column of 16 rows need 16 places
    constexpr int kTiles = kFormKeys / 32;
    __shared__ __attribute__((aligned(256))) uint8_t s_rows[kFormKeys * kLine];
    __shared__ __attribute__((aligned(16))) uint8_t s_out[kFormWaves][16 * 128];
    __shared__ uint32_t s_at[kFormKeys];
    __shared__ int32_t s_there[kFormKeys];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, half = lane >> 5;
    // Workgroups of neighbouring numbers are on different dies, each with an L2 of 4 MiB, and a head's matrices
    // take 256 KiB: a die goes through 8 heads or so, and all keys. (All heads on all dies: forming 12,800 keys of 32
    // heads took 206 us.) Within its heads, (tile of keys, pair of heads) units, in equal shares of neighbours.
    const int die = blockIdx.x % kDies, part = die % p.parts, all_pairs = (p.heads + 1) / 2;
    const int first = all_pairs * part / p.parts, pairs = all_pairs * (part + 1) / p.parts - first;
    const int workers = gridDim.x / p.parts, me = blockIdx.x / kDies * (kDies / p.parts) + die / p.parts;
    const int64_t units = (p.n_keys + kFormKeys - 1) / kFormKeys * pairs;
    const int64_t share1 = units * (me + 1) / workers;
    for (int64_t unit = units * me / workers; unit < share1;) {
    const int64_t tile = unit / pairs, key0 = tile * kFormKeys;
    const int from = (int)(unit - tile * pairs);
    const int until = pairs - from < share1 - unit ? pairs : from + (int)(share1 - unit);
    const int pair0 = first + from, pair1 = first + until;
    unit += until - from;
    __syncthreads();  // all are done with the tile before
    if (threadIdx.x < kFormKeys) {
        uint32_t at;
        const bool there = row_of(p, key0 + threadIdx.x, at);
        s_at[threadIdx.x] = at;
        s_there[threadIdx.x] = there;
        if (pair0 == 0 && key0 + threadIdx.x < p.n_keys) p.there[key0 + threadIdx.x] = there;
    }
    __syncthreads();
    const uint32_t lds = lds_of(s_rows);
    for (int i = 0; i < kFormKeys / kFormWaves; ++i) {
        const int j = wave * (kFormKeys / kFormWaves) + i;
        const uint8_t* const row = p.kv.rows + ((uint64_t)__builtin_amdgcn_readfirstlane(s_at[j]) << 4);
        if (L == 512 || lane < L / 8) fetch16(row, (uint32_t)lane * 16, lds + j * kLine);
    }
    if (pair0 == 0) {
        // the shared parts, 8 lanes a row
        for (int j = threadIdx.x / 8; j < kFormKeys; j += kFormThreads / 8) {
            if (key0 + j >= p.n_keys) break;
            const v4u x = *(const v4u*)(p.kv.rows + (((uint64_t)s_at[j] + L / 8 + threadIdx.x % 8) << 4));
            const v4u zero = {0u, 0u, 0u, 0u};
            *(v4u*)(p.rope + (key0 + j) * (kRope * 2) + threadIdx.x % 8 * 16) = s_there[j] ? x : zero;
        }
    }
    arrive<0>();
    __syncthreads();
    // rows that are not there are zeros
    for (int j = wave; j < kFormKeys; j += kFormWaves)
        if (!s_there[j] && lane < L / 8) *(v4u*)(s_rows + j * kLine + lane * 16) = v4u{0u, 0u, 0u, 0u};
    __syncthreads();

    const int last = 2 * pair1 < p.heads ? 2 * pair1 : p.heads;
    const bool value = wave & 2;  // of four waves the first two take a head's keys, the others its values
    const Rows& w = value ? p.wv : p.wk;
    // Rows 64 (wave & 1) .. of a head's matrix. Of each 64 latent values a lane takes 32 in a row, so that
    // whole lines are used; the keys are read to match.
    const int64_t next = w.token * 64;  // 32 rows on
    v4u x[2][8];  // this and the next 64 latent values of two rows
    auto load = [&](int head, int k, v4u (&to)[8]) {
        const uint8_t* const rows =
            (const uint8_t*)w.p + ((int64_t)head * w.head + (int64_t)((wave & 1) * 64 + n) * w.token + half * 32) * 2;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            to[s] = *(const v4u*)(rows + k * 128 + s * 16);
            to[4 + s] = *(const v4u*)(rows + next + k * 128 + s * 16);
        }
    };
    constexpr int kAtOnce = kFormWaves / 4;  // heads
    const int head0 = 2 * pair0 + (wave >> 2);
    if (head0 < last) load(head0, 0, x[0]);
    for (int head = head0; head < last; head += kAtOnce) {
        asm volatile("" ::: "memory");  // the keys stay in LDS: all of them do not fit the registers
        v16f o[2][kTiles];
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[a][t][e] = 0.f;
#pragma unroll
        for (int k = 0; k < L / 64; ++k) {
            if (k + 1 < L / 64) load(head, k + 1, x[(k + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);  // (or the loads move down to where registers are free)
            const v4u(&now)[8] = x[k & 1];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                V8 c[kTiles];
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
                    c[t] = __builtin_bit_cast(V8, *(const v4u*)(s_rows + (t * 32 + n) * kLine + k * 128 + half * 64 + s * 16));
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
                        o[a][t] = E::mma32(__builtin_bit_cast(V8, now[a * 4 + s]), c[t], o[a][t]);
            }
        }
        // the next head's first values, before the stores: a wait for loads waits for all stores before them
        if (head + kAtOnce < last) load(head + kAtOnce, 0, x[0]);
        // Out by way of LDS, 16 keys at a time, so that 8 lanes write a whole line of a key: straight from the
        // products' registers it is 32 bytes a key (forming 12,800 keys of 32 heads took 250 us so).
        uint8_t* const out = (value ? p.v : p.k) + ((int64_t)head * p.n_keys + key0) * kRow + (wave & 1) * 128;
        uint8_t* const mem = s_out[wave];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            v4u y[2][2][2];  // [nearest, left][tile of 32 values][16 of them]: 8 a lane
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int a = 0; a < 4; a += 2)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        // 4 values here, the next 4 in the other half: trade
                        uint32_t near[2], left[2];
#pragma unroll
                        for (int b = 0; b < 2; ++b)
                            near[b] = split2<kHalf>(o[i][t][4 * (a + b) + 2 * h], o[i][t][4 * (a + b) + 2 * h + 1], left[b]);
                        const auto x = __builtin_amdgcn_permlane32_swap(near[0], near[1], false, false);
                        y[0][i][a / 2][h] = x[0];
                        y[0][i][a / 2][2 + h] = x[1];
                        const auto w = __builtin_amdgcn_permlane32_swap(left[0], left[1], false, false);
                        y[1][i][a / 2][h] = w[0];
                        y[1][i][a / 2][2 + h] = w[1];
                    }
#pragma unroll
            for (int round = 0; round < 4; ++round) {
                const int kind = round & 1, up = round >> 1;  // nearest or left; which 16 keys
                if (n >> 4 == up) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        *(v4u*)(mem + (n & 15) * 128 + (((2 * c + half) ^ (n & 7)) * 16)) = y[kind][c >> 1][c & 1];
                }
                wave_order();
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int key = 8 * j + (lane >> 3), to = t * 32 + 16 * up + key;
                    const v4u x = *(const v4u*)(mem + key * 128 + (((lane & 7) ^ (key & 7)) * 16));
                    if (key0 + to < p.n_keys) 
                        __builtin_nontemporal_store(
                            x, (v4u*)(out + (int64_t)to * kRow + kind * (kRow / 2) + (lane & 7) * 16));
                }
                wave_order();
            }
        }
    }
    }
}

// The same of few keys: a workgroup takes 32 of them and the 128 rows of a head's keys or of its values, a wave 16 rows,
// all loads on their way at once. What such a call takes is the matrices' way to the compute units, about 40 GB/s
// each: spread over four times as many, 28 keys of 16 heads are formed in 8 us, not 25. Up to four workgroups
// a compute unit (3 prompts of up to 389 tokens, 16 heads, 53 us a call with both kernels, 57 by the one above; with
// eight, 2 prompts of up to 997 tokens 91, and 80).
template <int L, bool kHalf>
__global__ __launch_bounds__(kFormThreads) void k_form_few(ExpandedPlan p) {
    using E = Elem<kHalf>;
    using V8 = typename E::v8;
    constexpr int kLine = L * 2 + 16;  // bytes in LDS, as above
    constexpr int kOutLine = kRow + 16;
    static_assert(kValue == 16 * kFormWaves && kNope == kValue, "a wave takes 16 rows of a matrix");
    __shared__ __attribute__((aligned(256))) uint8_t s_rows[kFewKeys * kLine];
    __shared__ __attribute__((aligned(16))) uint8_t s_out[kFewKeys * kOutLine];
    __shared__ uint32_t s_at[kFewKeys];
    __shared__ int32_t s_there[kFewKeys];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, h4 = lane >> 4;
    const int units = 2 * p.heads;  // of a tile of keys
    const int64_t key0 = (int64_t)(blockIdx.x / units) * kFewKeys;
    const int unit = blockIdx.x % units, head = unit >> 1;
    const bool value = unit & 1;
    const Rows& w = value ? p.wv : p.wk;
    const uint8_t* const matrix =
        (const uint8_t*)w.p + ((int64_t)head * w.head + (int64_t)(wave * 16 + n) * w.token + h4 * 8) * 2;
    v4u x[L / 32];
#pragma unroll
    for (int k = 0; k < L / 32; ++k) x[k] = *(const v4u*)(matrix + k * 64);
    __builtin_amdgcn_sched_barrier(0);
    if (threadIdx.x < kFewKeys) {
        uint32_t at;
        const bool there = row_of(p, key0 + threadIdx.x, at);
        s_at[threadIdx.x] = at;
        s_there[threadIdx.x] = there;
        if (unit == 0 && key0 + threadIdx.x < p.n_keys) p.there[key0 + threadIdx.x] = there;
    }
    __syncthreads();
    const uint32_t lds = lds_of(s_rows);
#pragma unroll
    for (int i = 0; i < kFewKeys / kFormWaves; ++i) {
        const int j = wave * (kFewKeys / kFormWaves) + i;
        const uint8_t* const row = p.kv.rows + ((uint64_t)__builtin_amdgcn_readfirstlane(s_at[j]) << 4);
        if (L == 512 || lane < L / 8) fetch16(row, (uint32_t)lane * 16, lds + j * kLine);
    }
    const v4u zero = {0u, 0u, 0u, 0u};
    const int shared_row = threadIdx.x / 8, shared_at = threadIdx.x % 8 * 16;  // the shared parts, 8 lanes a row
    if (unit == 0 && shared_row < kFewKeys && key0 + shared_row < p.n_keys) {
        const v4u y = *(const v4u*)(p.kv.rows + (((uint64_t)s_at[shared_row] + L / 8) << 4) + shared_at);
        *(v4u*)(p.rope + (key0 + shared_row) * (kRope * 2) + shared_at) = s_there[shared_row] ? y : zero;
    }
    arrive<0>();
    // rows that are not there are zeros
#pragma unroll
    for (int i = 0; i < kFewKeys / kFormWaves; ++i) {
        const int j = wave * (kFewKeys / kFormWaves) + i;
        if (!s_there[j] && lane < L / 8) *(v4u*)(s_rows + j * kLine + lane * 16) = zero;
    }
    __syncthreads();
    v4f o[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};  // [16 values][16 keys]
#pragma unroll
    for (int k = 0; k < L / 32; ++k)
#pragma unroll
        for (int t = 0; t < 2; ++t)
            o[t] = E::mma16(__builtin_bit_cast(V8, x[k]),
                            __builtin_bit_cast(V8, *(const v4u*)(s_rows + (t * 16 + n) * kLine + k * 64 + h4 * 16)), o[t]);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        v2u near, left;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t rest;
            near[h] = split2<kHalf>(o[t][2 * h], o[t][2 * h + 1], rest);
            left[h] = rest;
        }
        uint8_t* const to = s_out + (t * 16 + n) * kOutLine + wave * 32 + h4 * 8;
        *(v2u*)to = near;
        *(v2u*)(to + kRow / 2) = left;
    }
    __syncthreads();
    uint8_t* const out = (value ? p.v : p.k) + ((int64_t)head * p.n_keys + key0) * kRow;
#pragma unroll
    for (int i = 0; i < kFewKeys * kRow / 16 / kFormThreads; ++i) {
        const int at = threadIdx.x + i * kFormThreads, key = at / (kRow / 16), c = at % (kRow / 16);
        if (key0 + key < p.n_keys) *(v4u*)(out + (int64_t)key * kRow + c * 16) = *(const v4u*)(s_out + key * kOutLine + c * 16);
    }
}

// Places in LDS: 16-byte column c of row r is at c ^ turn(r). K (and its shared part) is read by 16 lanes of
// 16 rows, one column; V by 32 lanes of 4 rows, 64 consecutive bytes each.
__device__ inline int turn_k(int row) { return row & 15; }
__device__ inline int turn_rope(int row) { return (row >> 1) & 7; }
__device__ inline int turn_v(int row) { return (row & 3) << 2; }  // (of a row's 32 columns, each 16 by themselves)

// As in prompt.hip: a running maximum that is behind by up to this much (in powers of two) is kept.
constexpr float kBehind = 8.f;
template <bool kHalf>
constexpr float kRoom = Elem<kHalf>::kRoom + (kHalf ? 0.f : kBehind);

// kSplit: 32 tokens a workgroup, whose waves take steps of keys in turn, each with an LDS buffer of its own and
// no barrier, and join what they found at the end: for calls that are a few steps' chain. kGroups 2: eight waves,
// the second four take every second step, in buffers of their own: for calls of one workgroup a compute unit.
template <bool kHalf, bool kSplit, int kGroups>
__global__ __launch_bounds__(kThreads * kGroups, kSplit || kGroups > 1 ? 1 : 2) void k_expanded(ExpandedPlan p) {
    using E = Elem<kHalf>;
    using V8 = typename E::v8;
    constexpr int kSteps = kNope / 16, kRopeSteps = kRope / 16, kTiles = kValue / 32;
    constexpr int kRopeRow = kRope * 2;  // bytes
    constexpr int kRopeAt = kKeys * kRow, kValueAt = kRopeAt + kKeys * kRopeRow, kBuffer = kValueAt + kKeys * kRow;
    static_assert(kNope * 4 == kRow && kValue * 4 == kRow, "rows of keys and of values are alike");
    constexpr int kTileRows = kSplit ? 32 : kPromptRows;
    __shared__ __attribute__((aligned(256))) uint8_t s_mem[(kSplit ? kWaves : 2 * kGroups) * kBuffer];
    __shared__ float s_max[kWaves][32], s_sum[kWaves][32];  // of the waves, where they join
    const int lane = threadIdx.x & 63, all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = all_waves % kWaves, group = all_waves / kWaves;
    const int n = lane & 31, half = lane >> 5;
    const int head = blockIdx.x % p.heads;
    // the last tiles of a request see the most keys: they go first
    const Tile f = find_tile(p, gridDim.x / p.heads - 1 - blockIdx.x / p.heads, kTileRows);
    if (f.tile < 0) return;

    // the request's packed keys: none where its offsets do not rise within 0 .. n_keys (compared before they are
    // subtracted, which of any two numbers could overflow)
    int64_t first = p.key_offsets[f.r], count = 0;
    const int64_t past_last = p.key_offsets[f.r + 1], limit = (int64_t)p.max_blocks * p.kv.div.page;
    if (first >= 0 && past_last >= first && past_last <= p.n_keys)
        count = past_last - first < limit ? past_last - first : limit;
    else
        first = 0;
    const int row0 = f.tile * kTileRows + (kSplit ? 0 : wave * 32);
    const int token = row0 + n < f.n ? row0 + n : f.n - 1;
    // (a row that sees no key, and one that sees them all, are at the ends of this range)
    auto clip = [&](int64_t x) { return (int32_t)(x < -1 ? -1 : (x < count ? x : count - 1)); };
    auto uniform = [&](int32_t x) { return __builtin_amdgcn_readfirstlane(x); };
    const int last_row = f.tile * kTileRows + kTileRows < f.n ? f.tile * kTileRows + kTileRows - 1 : f.n - 1;
    const int32_t end = uniform(clip(f.past + last_row) + 1);
    const int32_t tile_sees = uniform(clip(f.past + f.tile * kTileRows));
    const int32_t all_see = uniform(clip(f.past + (row0 < f.n ? row0 : f.n - 1)));
    const int32_t pos = clip(f.past + token);
    const int steps = (end + kKeys - 1) / kKeys;
    const uint8_t* const keys = p.k + ((int64_t)head * p.n_keys + first) * kRow;
    const uint8_t* const values = p.v + ((int64_t)head * p.n_keys + first) * kRow;
    const uint8_t* const shared = p.rope + first * kRopeRow;

    V8 q[kSteps + kRopeSteps];
    {
        const uint8_t* a = (const uint8_t*)p.qn.p + ((f.begin + token) * p.qn.token + head * p.qn.head) * 2;
        const uint8_t* b = (const uint8_t*)p.qr.p + ((f.begin + token) * p.qr.token + head * p.qr.head) * 2;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = __builtin_bit_cast(V8, *(const v4u*)(a + (s * 16 + half * 8) * 2));
#pragma unroll
        for (int s = 0; s < kRopeSteps; ++s)
            q[kSteps + s] = __builtin_bit_cast(V8, *(const v4u*)(b + (s * 16 + half * 8) * 2));
    }
    v16f o[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float top = kLowest, sum = 0.f;
    bool far = false;      // scores are scaled before the maximum is taken
    bool endless = false;  // a value that is not finite lies behind the first row's last key

    const uint32_t lds = lds_of(s_mem);
    // A step's rows 8 wave .. + 7 into LDS (a wave by itself: all 32), keys past the end as the last one.
    auto fetch = [&](int t, int buffer) {
        const int32_t at = t * kKeys, last = end - 1 - at;
        const uint32_t to = lds + buffer * kBuffer;
#pragma unroll
        for (int g = 0; g < (kSplit ? 4 : 1); ++g) {
            const int first_row = 8 * (kSplit ? g : wave);
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // two rows of 512 bytes
                const int j0 = first_row + 2 * i, j = j0 + half, key = j < last ? j : last;
                fetch16(keys + (int64_t)at * kRow, (uint32_t)(key * kRow + (n ^ turn_k(j)) * 16), to + j0 * kRow);
                fetch16(values + (int64_t)at * kRow, (uint32_t)(key * kRow + (n ^ turn_v(j)) * 16),
                        to + kValueAt + j0 * kRow);
            }
            const int j = first_row + (lane >> 3), key = j < last ? j : last;
            fetch16(shared + (int64_t)at * kRopeRow, (uint32_t)(key * kRopeRow + ((lane & 7) ^ turn_rope(j)) * 16),
                    to + kRopeAt + first_row * kRopeRow);
        }
    };
    // whether a lane's key of a step is there
    auto is_there = [&](int t) {
        const int32_t key = t * kKeys + n;
        return p.there[first + (key < end ? key : end - 1)];
    };
    // LDS places of a lane: see prompt.hip
    const int m8 = n >> 3, krow = 16 * (m8 >> 1) + 8 * ((n >> 2) & 1) + 4 * (m8 & 1) + (n & 3);
    uint32_t k_read[kSteps], r_read[kRopeSteps], v_read[kTiles];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) k_read[i] = krow * kRow + ((2 * i + half) ^ turn_k(krow)) * 16;
#pragma unroll
    for (int i = 0; i < kRopeSteps; ++i) r_read[i] = kRopeAt + krow * kRopeRow + ((2 * i + half) ^ turn_rope(krow)) * 16;
    {
        const int g = lane >> 4, l16 = lane & 15, row = 8 * (g >> 1) + (l16 >> 2);
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
            v_read[i] = kValueAt + row * kRow + ((4 * i + 2 * (g & 1) + ((l16 & 3) >> 1)) ^ turn_v(row)) * 16 + (l16 & 1) * 8;
    }

    int32_t flag = 0;
    if (!kSplit && group < steps) {
        flag = is_there(group);
        fetch(group, 2 * group);
    }
    for (int t0 = kSplit ? wave : 0; t0 < steps; t0 += kSplit ? kWaves : kGroups) {
        const int t = t0 + group, buf = kSplit ? wave : 2 * group + (t0 / kGroups & 1);
        const int32_t at = t * kKeys;
        if (kSplit) {
            flag = is_there(t);
            fetch(t, buf);
        }
        // the step is whole behind the barrier, and all waves are done with the other buffer
        arrive<0>();
        uint32_t ok = (uint32_t)__ballot(flag != 0 && at + n < end);
        asm volatile("" : "+s"(ok));  // (here, where nothing is under way: a wait for the flag costs nothing)
        if (!kSplit) {
            barrier();
            if (t + kGroups < steps) {
                flag = is_there(t + kGroups);
                fetch(t + kGroups, buf ^ 1);
            }
        }
        uint8_t* const mem = s_mem + buf * kBuffer;
        const int32_t last_key = (t0 + (kSplit ? 1 : kGroups)) * kKeys - 1;  // of the workgroup's steps
        if (last_key > tile_sees) {
            // Values that are not finite, in rows that the tile's first row does not see (a weight of zero would
            // make them NaN), become zeros. Every wave looks at all of them, so that all agree.
            bool found = false;
            const int j0 = at > tile_sees ? 0 : tile_sees + 1 - at;
            for (int g = 0; g < kGroups; ++g) {
                if (t0 + g >= steps) break;
                const int32_t from = (t0 + g) * kKeys;
                const uint8_t* const step = kGroups > 1 ? s_mem + (2 * g + (t0 / kGroups & 1)) * kBuffer : mem;
                const int32_t first_hidden = from > tile_sees ? 0 : tile_sees + 1 - from;
                for (int j = (kGroups > 1 ? first_hidden : j0) + (lane >> 4); j < kKeys; j += 4) {
                    v4u x = *(const v4u*)(step + kValueAt + j * kRow + (lane & 15) * 16);
                    found |= drop_endless<kHalf>(x);
                }
            }
            if (__any(found)) {
                endless = true;
                if (!kSplit) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                for (int j = j0 + (lane >> 4) + (kSplit ? 0 : 4 * wave); j < kKeys && t < steps; j += kSplit ? 4 : 16) {
                    v4u* const to = (v4u*)(mem + kValueAt + j * kRow + (lane & 15) * 16);
                    v4u x = *to;
                    if (drop_endless<kHalf>(x)) *to = x;
                }
                if (kSplit)
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                else
                    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            }
        }
        if (kGroups > 1 && t >= steps) break;  // (the last turn of the second four)
        v16f s;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * kSteps; ++i)
            s = E::mma32(__builtin_bit_cast(V8, *(const v4u*)(mem + k_read[i % kSteps] + i / kSteps * (kRow / 2))),
                         q[i % kSteps], s);
#pragma unroll
        for (int i = 0; i < kRopeSteps; ++i)
            s = E::mma32(__builtin_bit_cast(V8, *(const v4u*)(mem + r_read[i])), q[kSteps + i], s);
        // keys 16 (e >> 3) + 8 half + (e & 7) in s[e]
        if (ok != ~0u || at + kKeys - 1 > all_see) {
            // the keys that are there and that the row sees, from bit 0 those of s[0] on
            const int32_t ahead = pos - at;
            uint32_t seen = ahead < 0 ? 0 : (ahead > 30 ? ~0u : (2u << ahead) - 1);
            seen = (seen & ok) >> (8 * half);
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (!(seen & (1u << (16 * (e >> 3) + (e & 7))))) s[e] = -INFINITY;
        }
        float most = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) most = fmaxf(most, s[e]);
        most = larger_32(most);
        auto scale_now = [&] {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = product(s[e], p.scale2);
            most = product(most, p.scale2);
        };
        if (far) scale_now();
        float top2 = fmaxf(top, __builtin_fmaf(most, far ? 1.f : p.scale2, kRoom<kHalf>));
        if (__any(top2 > top + (far ? 0.f : kBehind))) {
            if (!far && __any(is_far(top2))) {
                far = true;
                scale_now();
                top2 = fmaxf(top, most + kRoom<kHalf>);
            }
            const float less = exp2_of(top - top2);
            sum *= less;
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[i][e] *= less;
            top = top2;
        }
        const float scale = far ? 1.f : p.scale2;
        v4u w[2];  // weights of 16 keys each, rounded to 16 bits as in prompt.hip; the sum takes them as they are
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = exp2_of(__builtin_fmaf(s[e], scale, -top));
            sum += s[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e >> 2][e & 3] = pack2<kHalf>(s[2 * e], s[2 * e + 1]);
#pragma unroll
        for (int b = 0; b < 4; ++b) {  // 16 keys; the nearest values, then what is left
            const uint32_t c = (b >> 1) * 16 * kRow + (b & 1) * (kRow / 2);
            v4u vt[kTiles];
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
                vt[i] = join(read_transposed(mem + v_read[i] + c), read_transposed(mem + v_read[i] + c + 4 * kRow));
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
                o[i] = E::mma32(__builtin_bit_cast(V8, vt[i]), __builtin_bit_cast(V8, w[b >> 1]), o[i]);
        }
        if (kSplit) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the step is read: the next may overwrite it
    }
    if (endless)
        for (int32_t key = tile_sees + 1; key < end; ++key) {
            if (key > pos || (kSplit && key / kKeys % kWaves != wave) || (kGroups > 1 && key / kKeys % kGroups != group))
                continue;
            const uint16_t* x = (const uint16_t*)(values + (int64_t)key * kRow);
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const uint16_t y = x[32 * i + 8 * (e >> 2) + 4 * half + (e & 3)];
                    o[i][e] = add_endless(o[i][e], kHalf ? (float)__builtin_bit_cast(_Float16, y)
                                                         : __uint_as_float((uint32_t)y << 16));
                }
        }
    if constexpr (kSplit) {
        sum += __shfl_xor(sum, 32);
        if (half == 0) {
            s_max[wave][n] = top;
            s_sum[wave][n] = sum;
        }
        __syncthreads();  // all are done with their steps, too
        float all = kLowest;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all = fmaxf(all, s_max[w][n]);
        const float less = exp2_of(top - all);
        float* const x = (float*)s_mem;  // [wave][dimensions / 4][row][4]
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *(v4f*)(x + ((wave * (kValue / 4) + 8 * i + 2 * a + half) * 32 + n) * 4) =
                    v4f{o[i][4 * a] * less, o[i][4 * a + 1] * less, o[i][4 * a + 2] * less, o[i][4 * a + 3] * less};
        __syncthreads();
        // a row and 16 dimensions a thread
        const int jr = threadIdx.x % 32, jc = threadIdx.x / 32, jt = f.tile * kTileRows + jr;
        if (jt >= f.n) return;
        all = kLowest;
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all = fmaxf(all, s_max[w][jr]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) total += exp2_of(s_max[w][jr] - all) * s_sum[w][jr];
        const float inv = total != 0.f ? 1.f / total : 0.f;
        uint8_t* const out = (uint8_t*)p.out.p + ((f.begin + jt) * p.out.token + head * p.out.head + jc * 16) * 2;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v4u y;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                v4f a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const v4f part = *(const v4f*)(x + ((w * (kValue / 4) + 4 * jc + 2 * h + b) * 32 + jr) * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[e] += part[e];
                }
                y[2 * b] = pack2<kHalf>(a[0] * inv, a[1] * inv);
                y[2 * b + 1] = pack2<kHalf>(a[2] * inv, a[3] * inv);
            }
            *(v4u*)(out + h * 16) = y;
        }
        if (p.lse && jc == 0)
            p.lse[(f.begin + jt) * p.heads + head] =
                total != 0.f ? (all + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
        return;
    }
    if constexpr (kGroups > 1) {
        // the second four's maxima, sums and outputs through LDS, lane by lane
        float* const x = (float*)s_mem + (wave * 64 + lane) * 4;
        __syncthreads();  // all are done with their steps
        if (group) {
            ((v2f*)s_mem)[kWaves * 64 * kTiles * 8 + wave * 64 + lane] = v2f{top, sum};
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int a = 0; a < 4; ++a)
                    *(v4f*)(x + (4 * i + a) * kWaves * 64 * 4) = v4f{o[i][4 * a], o[i][4 * a + 1], o[i][4 * a + 2], o[i][4 * a + 3]};
        }
        __syncthreads();
        if (group) return;
        const v2f other = ((const v2f*)s_mem)[kWaves * 64 * kTiles * 8 + wave * 64 + lane];
        const float all = fmaxf(top, other[0]), less = exp2_of(top - all), other_less = exp2_of(other[0] - all);
        sum = sum * less + other[1] * other_less;
        top = all;
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const v4f y = *(const v4f*)(x + (4 * i + a) * kWaves * 64 * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][4 * a + e] = o[i][4 * a + e] * less + y[e] * other_less;
            }
    }
    if (row0 + n >= f.n) return;  // both halves of a row leave together
    sum += __shfl_xor(sum, 32);
    // no key, or none with a weight: zeros, and the logarithm of nothing
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    uint8_t* const out = (uint8_t*)p.out.p + ((f.begin + token) * p.out.token + head * p.out.head) * 2;
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int a = 0; a < 4; a += 2) {
            v4u y;  // as in prompt.hip: 4 dimensions here, the next 4 in the other half
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t even = pack2<kHalf>(o[i][4 * a + 2 * h] * inv, o[i][4 * a + 2 * h + 1] * inv);
                const uint32_t odd = pack2<kHalf>(o[i][4 * a + 4 + 2 * h] * inv, o[i][4 * a + 4 + 2 * h + 1] * inv);
                const auto both = __builtin_amdgcn_permlane32_swap(even, odd, false, false);
                y[h] = both[0];
                y[2 + h] = both[1];
            }
            *(v4u*)(out + (32 * i + 8 * (a + half)) * 2) = y;
        }
    if (p.lse && half == 0)
        p.lse[(f.begin + token) * p.heads + head] =
            sum != 0.f ? (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f : -INFINITY;
}

template <int L, bool kHalf>
hipError_t run(const ExpandedPlan& p, int cus, hipStream_t s) {
    if (p.n_keys > 0) {
        const int64_t few = (p.n_keys + kFewKeys - 1) / kFewKeys * 2 * p.heads;
        if (few <= kFewTurns * cus) {
            hipLaunchKernelGGL((k_form_few<L, kHalf>), dim3((unsigned)few), dim3(kFormThreads), 0, s, p);
        } else {
            // one workgroup a compute unit, as LDS allows
            const int grid = (cus + kDies - 1) / kDies * kDies;
            hipLaunchKernelGGL((k_form<L, kHalf>), dim3((unsigned)grid), dim3(kFormThreads), 0, s, p);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    auto tiles = [&](int rows) { return p.R == 1 ? (p.n_tokens + rows - 1) / rows : tile_bound(p.n_tokens, 1, p.R, rows); };
    // Tiles of 32 where those of 128 leave half of the compute units idle: 2 prompts of up to 272 tokens, 8 heads,
    // 26 us a call (33), 500 tokens of 32 heads 53 (59); where they leave none, 1,000 tokens of 32 heads 101 (84).
    // Eight waves where a compute unit has one workgroup: 2,000 tokens of 16 heads 104 us (115), 1,000 of 32 79 (83);
    // 6 prompts of 33 to 3,500 tokens, several workgroups a compute unit, 415 (371).
    if (2 * tiles(kPromptRows) * p.heads <= cus)
        hipLaunchKernelGGL((k_expanded<kHalf, true, 1>), dim3((unsigned)(tiles(32) * p.heads)), dim3(kThreads), 0, s, p);
    else if (tiles(kPromptRows) * p.heads <= kGroupTurns * cus)
        hipLaunchKernelGGL((k_expanded<kHalf, false, 2>), dim3((unsigned)(tiles(kPromptRows) * p.heads)),
                           dim3(2 * kThreads), 0, s, p);
    else
        hipLaunchKernelGGL((k_expanded<kHalf, false, 1>), dim3((unsigned)(tiles(kPromptRows) * p.heads)), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

template <int L>
hipError_t run_kind(const ExpandedPlan& p, int cus, hipStream_t s) {
    return p.kv.kind == PTSTORE_KV_FP16 ? run<L, true>(p, cus, s) : run<L, false>(p, cus, s);
}

int64_t round16(int64_t x) { return (x + 15) / 16 * 16; }

}  // namespace

int64_t expanded_workspace(int32_t heads, int64_t n_keys) {
    return n_keys * heads * 2 * kRow + n_keys * kRope * 2 + round16(n_keys * 4);
}

void place_expanded(ExpandedPlan* p, void* workspace) {
    p->k = static_cast<uint8_t*>(workspace);
    p->v = p->k + p->n_keys * p->heads * kRow;
    p->rope = p->v + p->n_keys * p->heads * kRow;
    p->there = reinterpret_cast<int32_t*>(p->rope + p->n_keys * kRope * 2);
}

hipError_t launch_expanded(const ExpandedPlan& plan, int cus, hipStream_t s) {
    ExpandedPlan p = plan;
    for (p.parts = 1; p.parts < kDies && (int64_t)p.heads * 256 * p.kv.latent * 2 / p.parts > kDieBytes;) p.parts *= 2;
    return p.kv.latent == 512 ? run_kind<512>(p, cus, s) : run_kind<256>(p, cus, s);
}

}  // namespace ptsd
