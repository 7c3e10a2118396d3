// Attention in the latent space: a token's row is every head's key, and its latent part
// every head's value. Query rows are (token, head) pairs.
//
// A row of 1,152 bytes gives 4 * 512 + 2 * 64 operations a query row: with 16 heads a
// single token is bound by reading the rows, with 128 by the matrix units as much. The batch's
// work is cut into equal shares, as in decode.hip, one workgroup of eight waves a compute
// unit, for tiles of 128 query rows. Two waves take 32 rows, each one half of the dimensions: queries
// (72 registers) and outputs (128) stay in registers. Each sums its half of the scores, S^T = C Q^T; they
// trade these sums through LDS, form the same weights, and each its half of the output,
// O^T = C^T P^T (see attend.hpp). Waves whose rows do not exist only fetch. (A wave for 32 rows
// and all dimensions needs 400 registers, which the compiler spills.)
//
// Rows go from memory to LDS without passing through registers, 32 keys a piece, three pieces in
// turn, and are read there as they lie for the first product, transposed for the second.
//
// Measured: 32 requests of 128 heads, up to two tokens each behind 500 to 8,190, 70 us (39 GFLOP, 560 TFLOP/s; its two
// waves a SIMD wait at barriers and for memory 40 % of their time and to issue 31 %, matrix units 22 % of the cycles; then
// the parts' 80 MB) and 24 for the join; tiles of 16 rows: 64
// requests of 16 heads behind 120 to 8,190 tokens 67 us (309 MB, 4.6 TB/s; past its fixed 20 us it reads at 6.6), one
// of 777 tokens 14, and 8 and 6 for their joins.
#include <type_traits>

#include "attend.hpp"
#include "latent.hpp"
#include "lds_fetch.hpp"
#include "shares.hpp"

namespace ptsd {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr int kKeys = 32;    // of a piece
constexpr int kSpare = 8;    // pieces' time that a tile takes beside its keys
constexpr int kLeast = 2;    // steps of a share at least: a cut tile's parts are written and read again
// Pieces of a tile that is not cut: the share that it begins in takes all of it. 2 prompts of up to 45 tokens, 16 heads,
// 28 us a call (with none 31), 6 drafts of 64 heads 35 (40), 12 requests of 64 heads behind up to 1,025 tokens 34
// (32; with twelve pieces 43).
constexpr int kWhole = 4;
constexpr int kTile = 128;   // query rows
constexpr int kStages = 3;   // pieces in LDS: one is computed while two are on their way
constexpr int kAhead = kStages - 1;
constexpr int kEntries = 2 * kAhead + 2;  // pieces whose page entries are in LDS

// Floats of a part in the workspace: [4 dimensions][row], then rows' maxima and sums.
constexpr int part_floats(int latent, int tile) { return tile * (latent + 2); }

// A piece in LDS: rows' latent parts, padded by 16 bytes, row r in place place_of(r). 16 lanes read one
// 16-byte column of 16 rows as keys: all 16 places of 256 bytes. As values, 32 lanes read 64
// bytes of rows r .. r + 3, which are 4 places apart. And every address is a lane's own
// plus a constant: turned columns took a register for each. The shared parts, eight rows to a load, are not
// padded: 16-byte column c of row r is at c ^ turn_rope(r).
__device__ inline int place_of(int row) { return (row & 16) | (row & 3) << 2 | ((row >> 2) & 3); }
__device__ inline int turn_rope(int row) { return (row >> 1) & 7; }

// A running maximum that is behind by up to this much (in powers of two) is kept, as in prompt.hip.
constexpr float kBehind = 8.f;
template <bool kHalf>
constexpr float kRoom = Elem<kHalf>::kRoom + (kHalf ? 0.f : kBehind);

// Products 0 .. kProducts - 1 in groups of kDeep: the LDS reads of the next group are under way while one is
// computed. Left to itself the compiler, short of registers, reads and waits one by one.
template <int kDeep, int kProducts, class Read, class Multiply>
__device__ inline void pipelined(const Read& read, const Multiply& multiply) {
    v4u x[2][kDeep];
#pragma unroll
    for (int i = 0; i < kDeep; ++i) x[0][i] = read(i);
#pragma unroll
    for (int c = 0; c < kProducts; c += kDeep) {
        const int now = c / kDeep & 1;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kDeep; ++i)
            if (c + kDeep + i < kProducts) x[now ^ 1][i] = read(c + kDeep + i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kDeep; ++i)
            if (c + i < kProducts) multiply(c + i, x[now][i]);
    }
    __builtin_amdgcn_sched_barrier(0);
}

// A value that all lanes hold, in scalar registers.
__device__ inline int64_t uniform(int64_t x) {
    return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)x) |
           (int64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32;
}
__device__ inline Work uniform(const Work& w) {
    return {uniform(w.begin), __builtin_amdgcn_readfirstlane(w.n), uniform(w.past),
            __builtin_amdgcn_readfirstlane(w.steps), __builtin_amdgcn_readfirstlane(w.tiles)};
}

template <int L, bool kHalf>
__global__ __launch_bounds__(kThreads) void k_latent(LatentPlan p) {
    using E = Elem<kHalf>;
    using V8 = typename E::v8;
    constexpr int kSteps = L / 32, kRopeSteps = kRope / 32;  // of a half of the dimensions, 16 each
    constexpr int kTiles = L / 64;                           // of a half of the output, 32 dimensions each
    constexpr int kRow = L * 2 + 16;                         // bytes of a latent part in LDS
    constexpr int kPiece = kKeys * (kRow + kRope * 2);
    constexpr int kRows = kKeys / kWaves;                    // that a wave fetches of a piece
    constexpr int kFetches = kRows + 1;

    __shared__ __attribute__((aligned(256))) uint8_t s_rows[kStages * kPiece];
    __shared__ v4f s_score[kWaves][4 * 64];  // a wave's sums over its half
    __shared__ v4u s_query[kWaves][kRopeSteps * 64];  // the shared part of a wave's queries: registers are short
    __shared__ int32_t s_entry[kEntries * 64];
    __shared__ int s_endless;  // a value that is not finite lies behind the first row's last key

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int rg = wave >> 1, dh = wave & 1;  // rows, dimensions
    const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
    const int share = blockIdx.x;
    int r;
    int64_t first;  // the request's first step
    Work f;
    Shares shares = find_step<kTile, kWaves, kSpare, kLeast>(p, kKeys, share, false, r, f, first);
    shares = {uniform(shares.all), uniform(shares.count)};
    if (share >= shares.count) return;
    first = uniform(first);
    f = uniform(f);

    const uint32_t rows_at = lds_of(s_rows);
    const uint32_t entry_at = lds_of(s_entry);

    const int64_t share0 = shares.begin(share), share1 = shares.begin(share + 1);
    for (int64_t done = share0; done < share1;) {
    while (done >= first + f.all()) {  // on to the next request with work
        first += f.all();
        f = uniform(work_of<kTile, kSpare>(p, ++r, kKeys));
    }
    const int tile = (int)((done - first) / f.steps);
    const int64_t tile0 = first + (int64_t)tile * f.steps;  // the tile's first step
    const bool whole = f.steps <= kWhole + kSpare;
    if (whole && done > tile0) {  // the share before has it
        done = tile0 + f.steps;
        continue;
    }
    const int step0 = (int)(done - tile0);
    const int step1 = whole || share1 - tile0 >= f.steps ? f.steps : (int)(share1 - tile0);
    done = tile0 + step1;

    // the tile's rows see keys up to `end`; those of this share are [k0, k1)
    const int all_rows = f.n * p.group;
    const int row0 = tile * kTile + rg * 32;
    const bool active = row0 < all_rows;
    const int row = row0 + n < all_rows ? row0 + n : all_rows - 1;
    const int row_token = row / p.group, row_head = row - row_token * p.group;
    const int last_row = tile * kTile + kTile - 1 < all_rows ? tile * kTile + kTile - 1 : all_rows - 1;
    int64_t seen64 = f.past + last_row / p.group + 1;
    seen64 = seen64 < 0 ? 0 : (seen64 > limit ? limit : seen64);
    const int32_t end = __builtin_amdgcn_readfirstlane((int32_t)seen64);
    const int32_t k0 = step0 * kKeys;
    const int32_t k1 = end - k0 < (step1 - step0) * kKeys ? end : step1 * kKeys;
    const int64_t pos64 = f.past + row_token;  // the last key this lane's query sees
    const int32_t pos = pos64 < limit ? (int32_t)pos64 : (int32_t)limit;
    // the last key that the first row of the wave and of the tile sees
    auto clip = [&](int64_t x) { return __builtin_amdgcn_readfirstlane((int32_t)(x < limit ? x : limit)); };
    const int32_t all_see = clip(f.past + (active ? row0 : all_rows - 1) / p.group);
    const int32_t tile_sees = clip(f.past + tile * kTile / p.group);
    const int pieces = k1 > k0 ? (k1 - k0 + kKeys - 1) / kKeys : 0;
    const int32_t* const table = p.table + (int64_t)r * p.max_blocks;

    // queries: column n, 8 consecutive dimensions of each 16 a lane
    V8 q[kSteps];
    {
        const uint8_t* a = (const uint8_t*)p.ql.p + ((f.begin + row_token) * p.ql.token + row_head * p.ql.head) * 2 + dh * L;
        const uint8_t* b = (const uint8_t*)p.qr.p + ((f.begin + row_token) * p.qr.token + row_head * p.qr.head) * 2 + dh * kRope;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = __builtin_bit_cast(V8, *(const v4u*)(a + (s * 16 + half * 8) * 2));
#pragma unroll
        for (int s = 0; s < kRopeSteps; ++s) s_query[wave][s * 64 + lane] = *(const v4u*)(b + (s * 16 + half * 8) * 2);
    }
    v16f o[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float top = kLowest, sum = 0.f;
    bool far = false;      // scores are scaled before the maximum is taken

    // the page entries of a piece's keys into LDS (past the end: the last one's), by the first wave
    auto fetch_entries = [&](int piece, int lane) {
        if (wave) return;
        const int32_t key = k0 + piece * kKeys + (lane & 31), last = k1 - 1;
        fetch4_at(table + div_page((uint32_t)(key < last ? key : last), p.kv.div),
                  entry_at + (uint32_t)(piece % kEntries) * 256);
    };
    // a lane's key of a piece: its row, in units of 16 bytes, and whether it is there
    auto place = [&](int piece, int lane, bool& there) {
        const int32_t key = k0 + piece * kKeys + (lane & 31);
        const int32_t entry = s_entry[piece % kEntries * 64 + lane];
        there = key < k1 && entry >= 0 && entry < (int32_t)p.kv.blocks;
        const uint32_t slot = (uint32_t)key - div_page((uint32_t)key, p.kv.div) * p.kv.div.page;
        return there ? ((uint32_t)entry * p.kv.div.page + slot) * p.kv.line : 0u;
    };
    // this wave's rows of a piece into LDS
    auto fetch_rows = [&](int piece, int lane) {
        bool there;
        const uint32_t at = place(piece, lane, there);
        const uint32_t to = rows_at + (uint32_t)(piece % kStages) * kPiece;
        const int j0 = wave * kRows;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int j = j0 + i;
            const uint32_t row_at = (uint32_t)__builtin_amdgcn_readlane((int)at, j);
            const uint8_t* const row = p.kv.rows + ((uint64_t)row_at << 4);
            if (L == 512 || lane < L / 8) fetch16(row, (uint32_t)lane * 16, to + place_of(j) * kRow);
        }
        // the shared parts, 8 lanes a row
        const int mine = j0 + ((lane & 31) >> 3);
        const uint32_t a = (uint32_t)__builtin_amdgcn_ds_bpermute(mine * 4, (int)at);
        const int c = L / 8 + ((lane & 7) ^ turn_rope(mine));
        if (lane < 32) fetch16_at(p.kv.rows + (((uint64_t)a + c) << 4), to + kKeys * kRow + j0 * kRope * 2);
    };

    if (pieces > 0) {
        // (the tile before is done with all of LDS but s_endless, which is read behind its last barrier)
        barrier();
        int here = lane;
        asm volatile("" : "+v"(here));
        for (int i = 0; i <= kAhead; ++i) fetch_entries(i, here);
        if (threadIdx.x == 0) s_endless = 0;
        arrive<0>();
        barrier();
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {  // as in the loop's two turns before the first
            fetch_entries(kAhead + 1 + i, here);
            if (i < pieces) fetch_rows(i, here);
        }
    }
    for (int piece = 0; piece < pieces; ++piece) {
        // Behind the barrier the piece is whole, and all waves are done with the one before, whose
        // place the next to be fetched takes. Left under way: this wave's part of the next piece (and, so,
        // of page entries only those fetched after it, which are used three turns later).
        if (piece + 1 >= pieces)
            arrive<0>();
        else if (wave == 0)
            arrive<(kAhead - 1) * (kFetches + 1)>();
        else
            arrive<(kAhead - 1) * kFetches>();
        barrier();
        // what follows from the lane is formed anew each time: kept, it takes two dozen registers
        int here = lane;
        asm volatile("" : "+v"(here));
        fetch_entries(piece + kEntries - 1, here);
        if (piece + kAhead < pieces) fetch_rows(piece + kAhead, here);
        bool there;
        place(piece, here, there);
        const uint32_t ok = (uint32_t)__ballot(there);
        const uint8_t* const mem = s_rows + piece % kStages * kPiece;
        const int32_t at = k0 + piece * kKeys;

        // LDS places of a lane. As keys: the row that accumulator row n stands for, so that lanes then
        // hold 8 consecutive keys of each 16.
        const int n = here & 31, half = here >> 5;
        const int m8 = n >> 3, krow = 16 * (m8 >> 1) + 8 * ((n >> 2) & 1) + 4 * (m8 & 1) + (n & 3);
        const uint32_t k_read = place_of(krow) * kRow + dh * L + half * 16;
        const uint32_t r_read = kKeys * kRow + krow * kRope * 2 + ((4 * dh + half) ^ turn_rope(krow)) * 16;
        v16f s;
        if (active) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = 0.f;
            pipelined<3, kSteps + kRopeSteps>(
                [&](int i) {
                    const int j = i - kSteps;
                    return *(const v4u*)(mem + (j < 0 ? k_read + 32 * i : r_read ^ (32 * j)));
                },
                [&](int i, const v4u& x) {
                    const V8 y = i < kSteps ? q[i < kSteps ? i : 0] : __builtin_bit_cast(V8, s_query[wave][(i - kSteps) * 64 + here]);
                    s = E::mma32(__builtin_bit_cast(V8, x), y, s);
                });
#pragma unroll
            for (int a = 0; a < 4; ++a)
                s_score[wave][a * 64 + lane] = v4f{s[4 * a], s[4 * a + 1], s[4 * a + 2], s[4 * a + 3]};
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (ok != ~0u || at + kKeys - 1 > tile_sees) {
            // As values, rows that are not there become zeros, and so do values that are not finite where
            // the tile's first row does not see them: a weight of zero would make them NaN.
            bool endless = false;
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int j = wave * kRows + i;
                v4u* const x = (v4u*)(s_rows + piece % kStages * kPiece + place_of(j) * kRow) + lane;
                if (!((ok >> j) & 1)) {
                    if (lane < L / 8) *x = v4u{0u, 0u, 0u, 0u};
                } else if (at + j > tile_sees && lane < L / 8) {
                    v4u y = *x;
                    if (drop_endless<kHalf>(y)) {
                        endless = true;
                        *x = y;
                    }
                }
            }
            if (endless) s_endless = 1;
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
        if (!active) continue;
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const v4f x = s_score[wave ^ 1][a * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * a + e] += x[e];
        }

        // keys 16 (e >> 3) + 8 half + (e & 7) in s[e]
        const bool some_hidden = ok != ~0u || at + kKeys - 1 > all_see;
        if (some_hidden) {
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

        // as values: dimensions 16 (g & 1) .., keys 8 (g >> 1) .. of each 16, and those 4 further on
        const int g = here >> 4, l16 = here & 15, vrow = 8 * (g >> 1) + (l16 >> 2), vcol = 2 * (g & 1) + ((l16 & 3) >> 1);
        const uint32_t v_read = place_of(vrow) * kRow + dh * L + vcol * 16 + (l16 & 1) * 8;
        pipelined<2, 2 * kTiles>(
            [&](int j) {
                const int i = j % kTiles;
                const uint8_t* const x = mem + v_read + 64 * i + 16 * (j / kTiles) * kRow;
                return join(read_transposed(x), read_transposed(x + kRow));  // row + 4 is the next place
            },
            [&](int j, const v4u& x) {
                const int i = j % kTiles;
                o[i] = E::mma32(__builtin_bit_cast(V8, x), __builtin_bit_cast(V8, w[j / kTiles]), o[i]);
            });
    }
    sum += __shfl_xor(sum, 32);
    // loads of entries past the last piece may be under way; then every wave is done with its pieces
    arrive<0>();
    barrier();
    if (!active) continue;
    if (s_endless) {
        for (int32_t key = tile_sees + 1 > k0 ? tile_sees + 1 : k0; key < k1; ++key) {
            const int32_t entry = table[div_page((uint32_t)key, p.kv.div)];
            if (key > pos || entry < 0 || entry >= (int32_t)p.kv.blocks) continue;
            const uint32_t slot = (uint32_t)key - div_page((uint32_t)key, p.kv.div) * p.kv.div.page;
            int up = half;
            asm volatile("" : "+v"(up));  // no address is kept for this from before the pieces
            const uint16_t* x = (const uint16_t*)(p.kv.rows +
                ((uint64_t)(((uint32_t)entry * p.kv.div.page + slot) * p.kv.line) << 4)) + dh * (L / 2) + 4 * up;
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const uint16_t y = x[32 * i + 8 * (e >> 2) + (e & 3)];
                    o[i][e] = add_endless(o[i][e], kHalf ? (float)__builtin_bit_cast(_Float16, y)
                                                         : __uint_as_float((uint32_t)y << 16));
                }
        }
    }

    int column = n;
    asm volatile("" : "+v"(column));
    const int trow = rg * 32 + column;  // in the tile
    if (step0 > 0 || step1 < f.steps) {
        // a part: of a tile that began in an earlier share, or one that goes on
        float* const to = p.parts + (2 * (int64_t)share + (step0 > 0 ? 0 : 1)) * part_floats(L, kTile);
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *(v4f*)(to + ((L / 8 * dh + 8 * i + 2 * a + half) * kTile + trow) * 4) =
                    v4f{o[i][4 * a], o[i][4 * a + 1], o[i][4 * a + 2], o[i][4 * a + 3]};
        if (dh == 0 && half == 0) *(v2f*)(to + kTile * L + 2 * trow) = v2f{top, sum};
        continue;
    }
    if (row0 + column >= all_rows) continue;  // both halves of a row
    const int token = (row0 + column) / p.group, head = row0 + column - token * p.group;
    // no key, or none with a weight: zeros, and the logarithm of nothing
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    uint8_t* const out = (uint8_t*)p.out.p + ((f.begin + token) * p.out.token + head * p.out.head) * 2 + dh * L;
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int a = 0; a < 4; a += 2) {
            // 4 dimensions here, the next 4 in the other half: trade, and write 8 a lane
            v4u y;
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
    if (p.lse && dh == 0 && half == 0)
        p.lse[(f.begin + token) * p.group + head] =
            sum != 0.f ? (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f : -INFINITY;
    }
}

// Few rows: tiles of 16, and each of the eight waves takes pieces of 16 keys by itself, with all dimensions (72
// registers of queries, 128 of outputs), 128 keys of a share at a time, and no barrier until a tile's part is done.
// What a wave waits for memory the others fill. (As a pair of waves that trade scores and wait at barriers twice a
// piece, 64 requests of 16 heads took 82 us, not 67, where loading alone takes 50: a wave issues an instruction
// every five cycles or so, and a piece's chain of them was longer than its bytes take.)
constexpr int kFewRows16 = 16;
constexpr int kFewKeys = 16;                 // of a piece
constexpr int kFewStep = kWaves * kFewKeys;  // of a share's step
constexpr int kFewSpare = 2;                 // steps that a tile takes beside its keys
constexpr int kFewWhole = 1;                 // steps of a tile that is not cut

// A piece in LDS: rows' latent parts, padded by 16 bytes, row r in place few_place(r): 16 lanes that read a
// column of 16 rows find 16 places, and the 8 rows whose 32 bytes 32 lanes read as values are 32 bytes apart.
__device__ inline int few_place(int row) { return 2 * (row & 7) + (row >> 3); }

__device__ inline v4f mma16_few(v2u a, v2u b, v4f c, std::true_type) {
    typedef _Float16 v4 __attribute__((ext_vector_type(4)));
    return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(v4, a), __builtin_bit_cast(v4, b), c, 0, 0, 0);
}
__device__ inline v4f mma16_few(v2u a, v2u b, v4f c, std::false_type) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(v4s, a), __builtin_bit_cast(v4s, b), c, 0, 0, 0);
}

template <int L, bool kHalf>
__global__ __launch_bounds__(kThreads) void k_latent_few(LatentPlan p) {
    using E = Elem<kHalf>;
    using V8 = typename E::v8;
    constexpr int kTile = kFewRows16;
    constexpr int kSteps = L / 32, kRopeSteps = kRope / 32;  // of the first product, 32 dimensions each
    constexpr int kTiles = L / 16;                           // of the output, 16 dimensions each
    constexpr int kRow = L * 2 + 16;                         // bytes of a latent part in LDS
    constexpr int kPiece = kFewKeys * (kRow + kRope * 2);
    constexpr int kOut = 256;                                // dimensions that the waves join at once
    static_assert(kWaves * kTile * kOut * 4 <= kWaves * kPiece || L == 256, "");
    constexpr int kMem = kWaves * (kPiece > kTile * kOut * 4 ? kPiece : kTile * kOut * 4);

    __shared__ __attribute__((aligned(256))) uint8_t s_rows[kMem];
    __shared__ float s_max[kWaves][kTile], s_sum[kWaves][kTile];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, h4 = lane >> 4;  // query column, quarter
    const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
    const int share = blockIdx.x;
    int r;
    int64_t first;  // the request's first step
    Work f;
    Shares shares = find_step<kTile, kWaves, kFewSpare>(p, kFewStep, share, false, r, f, first);
    shares = {uniform(shares.all), uniform(shares.count)};
    if (share >= shares.count) return;
    first = uniform(first);
    f = uniform(f);
    uint8_t* const mem = s_rows + wave * kPiece;
    const uint32_t rows_at = lds_of(s_rows) + wave * kPiece;

    const int64_t share0 = shares.begin(share), share1 = shares.begin(share + 1);
    for (int64_t done = share0; done < share1;) {
    while (done >= first + f.all()) {  // on to the next request with work
        first += f.all();
        f = uniform(work_of<kTile, kFewSpare>(p, ++r, kFewStep));
    }
    const int tile = (int)((done - first) / f.steps);
    const int64_t tile0 = first + (int64_t)tile * f.steps;  // the tile's first step
    const bool whole = f.steps <= kFewWhole + kFewSpare;
    if (whole && done > tile0) {  // the share before has it
        done = tile0 + f.steps;
        continue;
    }
    const int step0 = (int)(done - tile0);
    const int step1 = whole || share1 - tile0 >= f.steps ? f.steps : (int)(share1 - tile0);
    done = tile0 + step1;

    // the tile's rows see keys up to `end`; those of this share are [k0, k1)
    const int all_rows = f.n * p.group;
    const int rows_left = all_rows - tile * kTile, rows = rows_left < kTile ? rows_left : kTile;
    const int row = tile * kTile + (n < rows ? n : rows - 1);
    const int token = row / p.group, head = row - token * p.group;
    int64_t seen64 = f.past + (tile * kTile + rows - 1) / p.group + 1;
    seen64 = seen64 < 0 ? 0 : (seen64 > limit ? limit : seen64);
    const int32_t end = __builtin_amdgcn_readfirstlane((int32_t)seen64);
    const int32_t k0 = step0 * kFewStep;
    const int32_t k1 = end - k0 < (step1 - step0) * kFewStep ? end : step1 * kFewStep;
    const int64_t pos64 = f.past + token;  // the last key this lane's query sees
    const int32_t pos = pos64 < limit ? (int32_t)pos64 : (int32_t)limit;
    const int64_t first64 = f.past + tile * kTile / p.group;
    const int32_t all_see = __builtin_amdgcn_readfirstlane(first64 < limit ? (int32_t)first64 : (int32_t)limit);
    const int32_t* const table = p.table + (int64_t)r * p.max_blocks;

    // queries: column n, 8 consecutive dimensions of each 32 a lane
    V8 q[kSteps + kRopeSteps];
    {
        const uint8_t* a = (const uint8_t*)p.ql.p + ((f.begin + token) * p.ql.token + head * p.ql.head) * 2;
        const uint8_t* b = (const uint8_t*)p.qr.p + ((f.begin + token) * p.qr.token + head * p.qr.head) * 2;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = __builtin_bit_cast(V8, *(const v4u*)(a + (s * 32 + h4 * 8) * 2));
#pragma unroll
        for (int s = 0; s < kRopeSteps; ++s)
            q[kSteps + s] = __builtin_bit_cast(V8, *(const v4u*)(b + (s * 32 + h4 * 8) * 2));
    }
    v4f o[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) o[i] = v4f{0.f, 0.f, 0.f, 0.f};
    float top = kLowest, sum = 0.f;
    bool far = false;      // scores are scaled before the maximum is taken
    bool endless = false;  // a value that is not finite lies behind the first row's last key

    auto entry_of = [&](int32_t key) {  // (past the end: the last one's)
        const int32_t last = k1 - 1;
        return table[div_page((uint32_t)(key < last ? key : last), p.kv.div)];
    };
    int32_t at = k0 + wave * kFewKeys;
    int32_t entry = at < k1 ? entry_of(at + n) : -1;
    for (; at < k1; at += kFewStep) {
        int here = lane;
        asm volatile("" : "+v"(here));  // what follows from the lane is formed anew each time
        const int n = here & 15, h4 = here >> 4;
        const int32_t key = at + n;
        const bool there = key < k1 && entry >= 0 && entry < (int32_t)p.kv.blocks;
        const uint32_t slot = (uint32_t)key - div_page((uint32_t)key, p.kv.div) * p.kv.div.page;
        const uint32_t place = there ? ((uint32_t)entry * p.kv.div.page + slot) * p.kv.line : 0u;
        const uint32_t ok = (uint32_t)__ballot(there) & 0xFFFFu;
#pragma unroll
        for (int j = 0; j < kFewKeys; ++j) {
            const uint32_t row_at = (uint32_t)__builtin_amdgcn_readlane((int)place, j);
            if (L == 512 || here < L / 8)
                fetch16_once(p.kv.rows + ((uint64_t)row_at << 4), (uint32_t)here * 16, rows_at + few_place(j) * kRow);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {  // the shared parts, 8 rows of 8 lanes
            const int j = 8 * i + (here >> 3);
            const uint32_t row_at = (uint32_t)__builtin_amdgcn_ds_bpermute(j * 4, (int)place);
            fetch16_at(p.kv.rows + (((uint64_t)row_at + L / 8 + ((here & 7) ^ turn_rope(j))) << 4),
                       rows_at + kFewKeys * kRow + i * 1024);
        }
        if (at + kFewStep < k1) entry = entry_of(at + kFewStep + n);
        arrive<0>();

        // S^T: row n of the piece as keys, 8 dimensions of each 32 a lane; keys 4 h4 + e in s[e]
        const uint8_t* const keys = mem + few_place(n) * kRow + h4 * 16;
        const uint8_t* const shared = mem + kFewKeys * kRow + n * (kRope * 2);
        v4f s = {0.f, 0.f, 0.f, 0.f};
        pipelined<3, kSteps + kRopeSteps>(
            [&](int i) {
                return *(const v4u*)(i < kSteps ? keys + 64 * i : shared + ((4 * (i - kSteps) + h4) ^ turn_rope(n)) * 16);
            },
            [&](int i, const v4u& x) { s = E::mma16(__builtin_bit_cast(V8, x), q[i], s); });
        const bool some_hidden = ok != 0xFFFFu || at + kFewKeys - 1 > all_see;
        if (some_hidden) {
            const int32_t ahead = pos - at;
            uint32_t seen = ahead < 0 ? 0 : (ahead > 14 ? ~0u : (2u << ahead) - 1);
            seen = (seen & ok) >> (4 * h4);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (!(seen & (1u << e))) s[e] = -INFINITY;
            // As values, rows that are not there become zeros, and so do values that are not finite where
            // the tile's first row does not see them: a weight of zero would make them NaN.
#pragma unroll 1
            for (int j = 0; j < kFewKeys; ++j) {
                v4u* const x = (v4u*)(mem + few_place(j) * kRow) + here;
                if (here >= L / 8) continue;
                if (!((ok >> j) & 1)) {
                    *x = v4u{0u, 0u, 0u, 0u};
                } else if (at + j > all_see) {
                    v4u y = *x;
                    if (drop_endless<kHalf>(y)) {
                        endless = true;
                        *x = y;
                    }
                }
            }
            wave_order();
        }
        float most = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
        most = larger_16_32(most);
        auto scale_now = [&] {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = product(s[e], p.scale2);
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
                for (int e = 0; e < 4; ++e) o[i][e] *= less;
            top = top2;
        }
        const float scale = far ? 1.f : p.scale2;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s[e] = exp2_of(__builtin_fmaf(s[e], scale, -top));
            sum += s[e];
        }
        // rounded to 16 bits as in prompt.hip; the sum takes them as they are
        const v2u w = {pack2<kHalf>(s[0], s[1]), pack2<kHalf>(s[2], s[3])};
        // O^T: 16 dimensions of 4 keys a quarter of the wave, read transposed
        const uint8_t* const values = mem + few_place(4 * h4 + (n >> 2)) * kRow + (n & 3) * 8;
        pipelined<4, kTiles>(
            [&](int i) {
                const v2u x = read_transposed(values + 32 * i);
                return v4u{x[0], x[1], 0u, 0u};
            },
            [&](int i, const v4u& x) {
                o[i] = mma16_few(v2u{x[0], x[1]}, w, o[i], std::integral_constant<bool, kHalf>{});
            });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the piece is read: the next may overwrite it
    }
    if (__any(endless)) {
        for (int32_t from = k0 + wave * kFewKeys; from < k1; from += kFewStep)
            for (int32_t key = from; key < k1 && key < from + kFewKeys; ++key) {
                if (key <= all_see || key > pos) continue;
                const int32_t entry = table[div_page((uint32_t)key, p.kv.div)];
                if (entry < 0 || entry >= (int32_t)p.kv.blocks) continue;
                const uint32_t slot = (uint32_t)key - div_page((uint32_t)key, p.kv.div) * p.kv.div.page;
                int up = h4;
                asm volatile("" : "+v"(up));  // no address is kept for this from before the pieces
                const uint16_t* x = (const uint16_t*)(p.kv.rows +
                    ((uint64_t)(((uint32_t)entry * p.kv.div.page + slot) * p.kv.line) << 4)) + 4 * up;
#pragma unroll
                for (int i = 0; i < kTiles; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint16_t y = x[16 * i + e];
                        o[i][e] = add_endless(o[i][e], kHalf ? (float)__builtin_bit_cast(_Float16, y)
                                                             : __uint_as_float((uint32_t)y << 16));
                    }
            }
    }

    // Join the eight waves: maxima and sums, then outputs at one scale, kOut dimensions at a time through LDS.
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    __syncthreads();  // the tile before is written
    if (h4 == 0) {
        s_max[wave][n] = top;
        s_sum[wave][n] = sum;
    }
    __syncthreads();
    const bool part = step0 > 0 || step1 < f.steps;
    float* const to = p.parts + (2 * (int64_t)share + (step0 > 0 ? 0 : 1)) * part_floats(L, kTile);
    {
        float all = kLowest;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all = fmaxf(all, s_max[w][n]);
        const float less = exp2_of(top - all);
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] *= less;
    }
    float* const x = (float*)s_rows;  // [wave][dimensions / 4][row][4]
#pragma unroll
    for (int c = 0; c < L; c += kOut) {
        __syncthreads();  // all are done with their pieces, or with what was joined before
#pragma unroll
        for (int i = 0; i < kOut / 16; ++i)
            *(v4f*)(x + ((wave * (kOut / 4) + 4 * i + h4) * kTile + n) * 4) = o[c / 16 + i];
        __syncthreads();
        // a row and 8 dimensions a thread
        const int jr = threadIdx.x % kTile, jc = threadIdx.x / kTile;
        float all = kLowest, total = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all = fmaxf(all, s_max[w][jr]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) total += exp2_of(s_max[w][jr] - all) * s_sum[w][jr];
        v4f a = {0.f, 0.f, 0.f, 0.f}, b = a;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const v4f y = *(const v4f*)(x + ((w * (kOut / 4) + 2 * jc) * kTile + jr) * 4);
            const v4f z = *(const v4f*)(x + ((w * (kOut / 4) + 2 * jc + 1) * kTile + jr) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] += y[e];
                b[e] += z[e];
            }
        }
        if (part) {
            // of a tile that began in an earlier share, or one that goes on
            *(v4f*)(to + ((c / 4 + 2 * jc) * kTile + jr) * 4) = a;
            *(v4f*)(to + ((c / 4 + 2 * jc + 1) * kTile + jr) * 4) = b;
            if (c == 0 && jc == 0) *(v2f*)(to + kTile * L + 2 * jr) = v2f{all, total};
        } else if (jr < rows) {
            // no key, or none with a weight: zeros, and the logarithm of nothing
            const float inv = total != 0.f ? 1.f / total : 0.f;
            const int out_row = tile * kTile + jr, ot = out_row / p.group, oh = out_row - ot * p.group;
            const v4u y = {pack2<kHalf>(a[0] * inv, a[1] * inv), pack2<kHalf>(a[2] * inv, a[3] * inv),
                           pack2<kHalf>(b[0] * inv, b[1] * inv), pack2<kHalf>(b[2] * inv, b[3] * inv)};
            *(v4u*)((uint8_t*)p.out.p + ((f.begin + ot) * p.out.token + oh * p.out.head + c + jc * 8) * 2) = y;
            if (p.lse && c == 0 && jc == 0)
                p.lse[(f.begin + ot) * p.group + oh] =
                    total != 0.f ? (all + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
        }
    }
    __syncthreads();  // the next tile's pieces go there
    }
}

// Joins the parts of a tile that several shares have: the workgroups of all these shares but the last, kGroupsOf
// each (64 requests of 16 heads: 78 us a call with two, 82 with four; 32 of 128 heads 96 and 91), take its (row, 8
// dimensions) items in turn. A lane loads eight parts at once; where a tile has more, several lanes divide
// them, so that each has few trips to memory.
constexpr int kJoinThreads = 512;
constexpr int kJoinGroups = 4, kFewJoinGroups = 2;  // of a tile of 128, and of 16 rows

// A row's parts so far: 8 dimensions of the output, the maximum, the sum.
struct Joined {
    v4f acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    float all = kLowest, total = 0.f;
    // To a maximum of at least `top`. Sums that then weigh nothing stay in, and are NaN where they are not
    // finite: a part whose scores are all NaN has the lowest maximum.
    __device__ void raise(float top) {
        const float to = fmaxf(all, top), less = exp2_of(all - to);
        total *= less;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[h][e] *= less;
        all = to;
    }
    // a part whose maximum is not above `all`
    __device__ void add(v4f a, v4f b, float top, float sum) {
        const float part_of = exp2_of(top - all);
        total += part_of * sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            acc[0][e] += part_of * a[e];
            acc[1][e] += part_of * b[e];
        }
    }
};

template <int L, bool kHalf, int kTile, int kStep, int kSpareOf, int kLeastOf, int kWholeOf, int kGroupsOf>
__global__ __launch_bounds__(kJoinThreads) void k_latent_join(LatentPlan p) {
    constexpr int kFlight = 8;
    __shared__ v4f s_acc[2][kJoinThreads];
    __shared__ float s_all[kJoinThreads], s_total[kJoinThreads];
    int r;
    int64_t first;
    Work f;
    const int share = blockIdx.x / kGroupsOf;
    const Shares shares = find_step<kTile, kJoinThreads / 64, kSpareOf, kLeastOf>(p, kStep, share, true, r, f, first);
    if (share >= shares.count || f.steps <= kWholeOf + kSpareOf) return;
    const int64_t share1 = shares.begin(share + 1);
    const int tile = (int)((share1 - 1 - first) / f.steps);
    const int64_t tile0 = first + (int64_t)tile * f.steps, tile1 = tile0 + f.steps;
    if (tile1 <= share1) return;
    const int share0 = (int)shares.of(tile0);  // the tile's first
    const int parts = (int)(shares.of(tile1 - 1) - share0 + 1);
    const int rows_left = f.n * p.group - tile * kTile, rows = rows_left < kTile ? rows_left : kTile;
    const int items = rows * (L / 8);
    int slices = 1;  // lanes that divide an item's parts
    while (slices < 32 && slices * kFlight < parts) slices *= 2;
    const int at_once = kJoinThreads / slices;
    const int slice = threadIdx.x / at_once, lane_item = threadIdx.x % at_once;
    // the first share's second part, then the first of each following
    const float* const from = p.parts + (2 * (int64_t)share0 + 1) * part_floats(L, kTile);
    auto part_at = [&](int i) { return from + (int64_t)(2 * i - (i > 0)) * part_floats(L, kTile); };
    const int me = (share - share0) * kGroupsOf + blockIdx.x % kGroupsOf, workers = (parts - 1) * kGroupsOf;
    for (int item0 = me * at_once; item0 < items; item0 += workers * at_once) {
        const int item = item0 + lane_item < items ? item0 + lane_item : items - 1;
        const int trow = item % rows, c = item / rows;
        Joined sum;
        for (int i0 = slice; i0 < parts; i0 += slices * kFlight) {
            v4f a[kFlight], b[kFlight];
            v2f ms[kFlight];
#pragma unroll
            for (int u = 0; u < kFlight; ++u) {
                const int i = i0 + u * slices;
                const float* part = part_at(i < parts ? i : i0);
                ms[u] = *(const v2f*)(part + kTile * L + 2 * trow);
                a[u] = *(const v4f*)(part + (2 * c * kTile + trow) * 4);
                b[u] = *(const v4f*)(part + ((2 * c + 1) * kTile + trow) * 4);
                if (i >= parts) {
                    ms[u] = v2f{-INFINITY, 0.f};
                    a[u] = b[u] = v4f{0, 0, 0, 0};
                }
            }
            float top = kLowest;
#pragma unroll
            for (int u = 0; u < kFlight; ++u) top = fmaxf(top, ms[u][0]);
            sum.raise(top);
#pragma unroll
            for (int u = 0; u < kFlight; ++u) sum.add(a[u], b[u], ms[u][0], ms[u][1]);
        }
        if (slices > 1) {
            __syncthreads();
            s_acc[0][threadIdx.x] = sum.acc[0];
            s_acc[1][threadIdx.x] = sum.acc[1];
            s_all[threadIdx.x] = sum.all;
            s_total[threadIdx.x] = sum.total;
            __syncthreads();
            if (slice == 0)
                for (int i = 1; i < slices; ++i) {
                    const int t = i * at_once + lane_item;
                    sum.raise(s_all[t]);
                    sum.add(s_acc[0][t], s_acc[1][t], s_all[t], s_total[t]);
                }
        }
        if (item0 + lane_item >= items || slice) continue;
        const int row = tile * kTile + trow, token = row / p.group, head = row - token * p.group;
        const float total = sum.total, inv = total != 0.f ? 1.f / total : 0.f;
        v4u y;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y[e] = pack2<kHalf>(sum.acc[e >> 1][2 * (e & 1)] * inv, sum.acc[e >> 1][2 * (e & 1) + 1] * inv);
        *(v4u*)((uint8_t*)p.out.p + ((f.begin + token) * p.out.token + head * p.out.head + c * 8) * 2) = y;
        if (p.lse && c == 0)
            p.lse[(f.begin + token) * p.group + head] =
                total != 0.f ? (sum.all + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
    }
}

template <int L, bool kHalf, int kTile, int kStep, int kSpareOf, int kLeastOf, int kWholeOf, int kGroupsOf>
hipError_t join(const LatentPlan& p, hipStream_t s) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_latent_join<L, kHalf, kTile, kStep, kSpareOf, kLeastOf, kWholeOf, kGroupsOf>), dim3((unsigned)(p.shares * kGroupsOf)),
                       dim3(kJoinThreads), 0, s, p);
    return hipGetLastError();
}

// Tiles of 16 rows where that leaves a request one of them: the host knows the average request alone.
template <int L, bool kHalf>
hipError_t run(const LatentPlan& p, hipStream_t s) {
    if (p.n_tokens * p.group <= (int64_t)kFewRows16 * p.R) {
        hipLaunchKernelGGL((k_latent_few<L, kHalf>), dim3((unsigned)p.shares), dim3(kThreads), 0, s, p);
        return join<L, kHalf, kFewRows16, kFewStep, kFewSpare, 1, kFewWhole, kFewJoinGroups>(p, s);
    }
    hipLaunchKernelGGL((k_latent<L, kHalf>), dim3((unsigned)p.shares), dim3(kThreads), 0, s, p);
    return join<L, kHalf, kTile, kKeys, kSpare, kLeast, kWhole, kJoinGroups>(p, s);
}

template <int L>
hipError_t run_kind(const LatentPlan& p, hipStream_t s) {
    return p.kv.kind == PTSTORE_KV_FP16 ? run<L, true>(p, s) : run<L, false>(p, s);
}

}  // namespace

// One workgroup a compute unit, two parts each.
int64_t latent_workspace(int latent, int cus) {
    return 2ll * cus * part_floats(latent, kTile) * (int64_t)sizeof(float);
}

hipError_t launch_latent(const LatentPlan& p, hipStream_t s) {
    return p.kv.latent == 512 ? run_kind<512>(p, s) : run_kind<256>(p, s);
}

}  // namespace ptsd
