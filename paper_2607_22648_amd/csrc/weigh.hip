// The attention weights that a batch's queries gave to each cached token, added to what it had:
//   weight(j) += sum over rows that see key j of exp(scale q . k_j - lse).
//
// S = Q K^T, 16 x 16 at a time with keys as columns: a lane holds one key's scores of 4 rows, so that
// sums over rows stay in the lane, and no weight is ever rounded. Few rows are bound by reading K once;
// many by the exponentials and what else is vector instructions (an exponential is 16 cycles of a wave for 64, as long
// as 2 dim operations of a row take for dim 128) and by the matrix units: two waves a SIMD overlap them in part.
//
// A workgroup of four waves takes a tile of keys, 64 a wave (32 of a latent cache), as registers of the
// second factor, and goes through the query rows that see it, 32 at a time, which pass through LDS for
// all four. Where 32 are all that a request has they stay there, and the waves go from tile to tile by
// themselves. (Key tile, 32 rows) items of the batch, those above the diagonal left out, are laid end to end and
// cut into equal shares, as decode.hip's steps; a tile of more than 4 (16) items may be cut, and a second kernel
// adds what its shares found, in order: the same inputs give the same bits.
//
// Measured: a step of 64 requests of 120 to 8,190 tokens, 8 heads of 128, 93 us (562 MB, 6.0 TB/s); of 32 over latent
// rows 34 (4.5 TB/s: 16 rows are a load, whose 64 lanes take 64-byte pieces); prompts of 128 to 1,500 tokens over 4 bits
// 96 (matrix units 27 % of the cycles, other vector instructions 44). A step over 4-bit pages, the 64 requests' above,
// 59 a call, by loads of lanes; prompts over 16 bits 100.
#include <type_traits>

#include "attend.hpp"
#include "lds_fetch.hpp"
#include "shares.hpp"
#include "weights.hpp"

namespace ptsd {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kRowsOf = 32;  // query rows of an item
constexpr int kLatent = 2;   // kinds of keys: 16 bits, 4 bits, latent rows

constexpr int keys_of(int layout) { return kWaves * (layout == kLatent ? 32 : 64); }  // of a tile

// A request's items. Its key tiles 0 .. seen + 1 - 1 are seen by all row tiles; tile seen + i by those from
// i * rise - late on (i >= 1): a tile's keys are a whole number of row tiles.
struct Items {
    int64_t begin;  // first token that has a position
    int32_t n;
    int32_t past;
    int32_t tiles, rows, seen;
    int64_t rise, late;
    // items before tile t
    __device__ int64_t before(int64_t t) const {
        const int64_t j = t - 1 - seen;
        return t * rows - (j > 0 ? rise * (j * (j + 1) / 2) - late * j : 0);
    }
    __device__ int64_t all() const { return before(tiles); }
    __device__ int32_t first_row(int32_t t) const {
        const int64_t i = t - seen;
        return i > 0 ? (int32_t)(i * rise - late) : 0;
    }
};

// stream: of a request that has one row tile, and the others have none; else of the others, and where nothing else
// takes those of one row tile, of them, too
__device__ inline Items items_of(const WeighPlan& p, int r, int keys, bool stream) {
    Items w;
    int64_t a = p.offsets[r], b = p.offsets[r + 1];
    const bool ok = a >= 0 && b > a && b <= p.n_tokens;
    int64_t past = p.context[r];
    if (past < 0) {  // tokens before position 0 see nothing
        a -= past;
        past = 0;
    }
    w.begin = a;
    w.n = ok && b > a ? (int32_t)(b - a) : 0;
    w.past = (int32_t)past;
    const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
    int64_t end = past + w.n;
    end = w.n == 0 ? 0 : end > limit ? limit : end;
    w.tiles = (int32_t)((end + keys - 1) / keys);
    w.rows = (int32_t)(((int64_t)w.n * p.group + kRowsOf - 1) / kRowsOf);
    if (stream ? w.rows != 1 : w.rows == 1 && p.apart) w.tiles = 0;
    w.seen = (int32_t)(past / keys);
    w.rise = (int64_t)(keys / kRowsOf) * p.group;
    w.late = (past % keys * p.group + kRowsOf - 1) / kRowsOf;
    return w;
}

// The tile that item y is in.
__device__ inline int32_t tile_of(const Items& f, int64_t y) {
    int32_t lo = 0, span = f.tiles;
    while (span > 1) {
        const int32_t half = span / 2;
        if (f.before(lo + half) <= y) {
            lo += half;
            span -= half;
        } else {
            span = half;
        }
    }
    return lo;
}

// A key's slot of the weights, or -1.
__device__ inline int64_t weight_at(const WeighPlan& p, int r, int head, int64_t key) {
    const uint32_t column = div_page((uint32_t)key, p.kv.div);
    const int32_t entry = p.table[(int64_t)r * p.max_blocks + column];
    if (entry < 0 || entry >= p.kv.blocks) return -1;
    return ((int64_t)entry * p.kv.heads + head) * p.kv.div.page + ((uint32_t)key - column * p.kv.div.page);
}

__device__ inline void put_weight(const WeighPlan& p, int r, int head, int32_t key, float sum) {
    const int64_t at = weight_at(p, r, head, key);
    if (at < 0) return;
    const int32_t had = p.weighed ? p.weighed[r] : p.context[r];
    p.weights[at] = key < had ? p.weights[at] + sum : sum;
}

// Waves of a SIMD: as many as the registers hold.
constexpr int weigh_waves(int dim) { return dim == 576 ? 2 : 3; }

// kDim: of a row; kLayout: how keys are kept; kStream: requests of one row tile, else those of several.
template <int kDim, int kLayout>
struct WeighShape {
    static constexpr int kColumns = kDim / 8;  // 16-byte columns of a row
    // Rows in LDS are padded by a column, so that 16 lanes which read one column of 16 rows find 16 places; the
    // shared parts of latent queries, which come eight rows to a load, are turned instead.
    static constexpr int kOwn = kLayout == kLatent ? kColumns - kRope / 8 : kColumns;  // columns before the shared part
    static constexpr int kRow = kOwn * 16 + 16, kRopeRow = kRope * 2;
    static constexpr int kBuffer = kRowsOf * (kRow + (kLayout == kLatent ? kRopeRow : 0));
};

template <int kDim, bool kHalf, int kLayout, bool kStream>
__device__ inline void weigh(const WeighPlan& p, int block, uint8_t (&s_q)[2][WeighShape<kDim, kLayout>::kBuffer],
                             float (&s_lse)[2][kRowsOf]) {
    using Shape = WeighShape<kDim, kLayout>;
    using E = Elem<kHalf>;
    using V8 = typename E::v8;
    constexpr bool kFour = kLayout == 1;
    constexpr int kTile = keys_of(kLayout), kGroups = kTile / kWaves / 16;  // of a wave, 16 keys each
    constexpr int kSteps = kDim / 32, kColumns = Shape::kColumns;  // matrix steps
    constexpr int kOwn = Shape::kOwn, kRow = Shape::kRow, kRopeRow = Shape::kRopeRow;
    constexpr int kPieces = kLayout == kLatent ? 1 : kRowsOf * kColumns / kThreads;  // of queries, a thread

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, h4 = lane >> 4;  // key column, quarter
    const int head = block % p.kv.heads, share = block / p.kv.heads;
    int r;
    int64_t first;
    Items f;
    const Shares shares = find_share<kWaves>(
        p.R, kStream ? p.streams : p.shares, [&](int i) { return items_of(p, i, kTile, kStream); }, share, false, r, f, first);
    if (share >= shares.count) return;
    const int64_t share0 = shares.begin(share), share1 = shares.begin(share + 1);
    for (int64_t done = share0; done < share1;) {
        while (done >= first + f.all()) {
            first += f.all();
            f = items_of(p, ++r, kTile, kStream);
        }
        const int32_t tile = kStream ? (int32_t)(done - first) : tile_of(f, done - first);
        const int64_t tile0 = kStream ? done : first + f.before(tile), tile1 = kStream ? done + 1 : first + f.before(tile + 1);
        if (!kStream && f.rows <= p.whole && done > tile0) {  // the share before has all of it
            done = tile1;
            continue;
        }
        const int32_t row_first = kStream ? 0 : f.first_row(tile);
        const int32_t rt0 = row_first + (int32_t)(done - tile0);
        const int64_t stop = f.rows <= p.whole || tile1 < share1 ? tile1 : share1;
        const int32_t rt1 = row_first + (int32_t)(stop - tile0);
        const bool part = done > tile0 || stop < tile1;
        float* const to = p.parts + (2 * (int64_t)block + (done > tile0 ? 0 : 1)) * kTile;
        done = stop;

        const int64_t limit64 = (int64_t)p.max_blocks * p.kv.div.page;
        const int64_t end64 = (int64_t)f.past + f.n < limit64 ? (int64_t)f.past + f.n : limit64;
        const int32_t end = (int32_t)end64;
        const int32_t k0 = tile * kTile + wave * (16 * kGroups);
        const int all_rows = f.n * p.group;
        const int32_t* const table = p.table + (int64_t)r * p.max_blocks;
        const int32_t had = p.weighed ? p.weighed[r] : p.context[r];  // tokens that have weights

        // Keys: column n of a group; 8 consecutive values of each 32 a lane, or (4 bits) a quarter of the row. Four
        // lanes so read 64 bytes of a row at once.
        auto entry_of = [&](int32_t key) {
            return table[div_page((uint32_t)(key < end ? key : end - 1), p.kv.div)];
        };
        auto slot_of = [&](int32_t key) { return (uint32_t)key - div_page((uint32_t)key, p.kv.div) * p.kv.div.page; };
        auto is_there = [&](int32_t entry, int32_t key) {
            return key < end && entry >= 0 && entry < (int32_t)p.kv.blocks;
        };
        auto load_key = [&](V8 (&to)[kSteps], int32_t entry, int32_t key) {
            const bool there = is_there(entry, key);
            const uint32_t page = there ? (uint32_t)entry : 0u, slot = there ? slot_of(key) : 0u;
            const uint32_t line = head * p.kv.div.page + slot;
            if constexpr (kFour) {
                const uint8_t* row = p.kv.k + (uint64_t)page * p.kv.slab + (uint64_t)line * (kDim / 2) + h4 * (kDim / 8);
                const float step = step_of(p.kv.k[(uint64_t)page * p.kv.slab + p.kv.exponents +
                                                  (uint64_t)line * (kDim / kGroup) + h4 * (kDim / 4) / kGroup]);
                uint32_t codes[kSteps];
                if constexpr (kSteps == 4)
                    *(v4u*)codes = *(const v4u*)row;
                else
                    *(v2u*)codes = *(const v2u*)row;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) to[i] = __builtin_bit_cast(V8, widen8(codes[i], step));
            } else {
                const uint8_t* row =
                    kLayout == kLatent
                        ? p.latent.rows + ((uint64_t)((page * p.kv.div.page + slot) * p.latent.line) << 4)
                        : p.kv.k + (uint64_t)page * p.kv.slab + (uint64_t)line * (kDim * 2);
#pragma unroll
                for (int i = 0; i < kSteps; ++i) to[i] = __builtin_bit_cast(V8, *(const v4u*)(row + (4 * i + h4) * 16));
            }
        };
        auto weight_of = [&](int32_t entry, int32_t key) {
            return p.weights + ((int64_t)entry * p.kv.heads + head) * p.kv.div.page + slot_of(key);
        };

        V8 k[kGroups][kSteps];
        int32_t entry[kGroups];
        if constexpr (!kStream) {
#pragma unroll
            for (int c = 0; c < kGroups; ++c) entry[c] = entry_of(k0 + 16 * c + n);
#pragma unroll
            for (int c = 0; c < kGroups; ++c) load_key(k[c], entry[c], k0 + 16 * c + n);
        }

        v4u piece[kPieces];
        float lse = 0.f;
        // a tile of query rows on its way to LDS, by registers, a latent cache's straight there (its rows would take
        // 36 registers); rows past the last one as the last
        auto load = [&](int rt, int buffer) {
            auto place = [&](int j, int& token, int& sub) {
                const int row = rt * kRowsOf + j < all_rows ? rt * kRowsOf + j : all_rows - 1;
                token = (int)div_page((uint32_t)row, p.rows_div);
                sub = row - token * p.group;
            };
            int token, sub;
            if constexpr (kLayout == kLatent) {
                place(lane & 31, token, sub);
                const int64_t own = (f.begin + token) * p.q.token + (int64_t)sub * p.q.head;
                const int64_t shared = (f.begin + token) * p.qr.token + (int64_t)sub * p.qr.head;
                const uint32_t to = lds_of(s_q[buffer]);
#pragma unroll
                for (int i = 0; i < kRowsOf / kWaves; ++i) {
                    const int j = wave * (kRowsOf / kWaves) + i;
                    const int64_t at = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)own, j) |
                                       (int64_t)__builtin_amdgcn_readlane((int)(own >> 32), j) << 32;
                    if (lane < kOwn) fetch16((const uint8_t*)p.q.p + at * 2, (uint32_t)lane * 16, to + j * kRow);
                }
                const int j = wave * 8 + (lane >> 3);
                const int64_t at = (int64_t)(uint32_t)__builtin_amdgcn_ds_bpermute(4 * j, (int)shared) |
                                   (int64_t)__builtin_amdgcn_ds_bpermute(4 * j, (int)(shared >> 32)) << 32;
                fetch16_at((const uint8_t*)p.qr.p + at * 2 + ((lane & 7) ^ ((j >> 1) & 7)) * 16,
                           to + kRowsOf * kRow + wave * 8 * kRopeRow);
            } else {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int at = threadIdx.x + i * kThreads, c = at % kColumns;
                    place(at / kColumns, token, sub);
                    piece[i] = *(const v4u*)((const uint8_t*)p.q.p + ((f.begin + token) * p.q.token +
                                                                     (int64_t)(head * p.group + sub) * p.q.head) * 2 + c * 16);
                }
            }
            if (threadIdx.x < kRowsOf) {
                place(threadIdx.x, token, sub);
                lse = rt * kRowsOf + (int)threadIdx.x < all_rows
                          ? p.lse[(f.begin + token) * p.q_heads + head * p.group + sub] : -INFINITY;
                // rows that saw no key, and those that do not exist, give nothing: a weight of 2^-inf
                lse = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f;
            }
        };
        auto store = [&](int buffer) {
            if constexpr (kLayout != kLatent) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int at = threadIdx.x + i * kThreads, j = at / kColumns, c = at % kColumns;
                    *(v4u*)(s_q[buffer] + j * kRow + c * 16) = piece[i];
                }
            }
            if (threadIdx.x < kRowsOf) s_lse[buffer][threadIdx.x] = lse;
            if (kLayout == kLatent) arrive<0>();
        };

        // Adds to `sum` what row tile rt gives to the keys of kOf groups from `key0` on.
        auto rows_of = [&](auto groups, const V8 (*k)[kSteps], int32_t key0, int32_t rt, int buffer, float* sum) {
            constexpr int kOf = decltype(groups)::value;
#pragma unroll
            for (int up = 0; up < 2; ++up) {
                const int row0 = rt * kRowsOf + 16 * up;
                if (up && row0 >= all_rows) break;
                const uint8_t* const mem = s_q[buffer] + (n + 16 * up) * kRow;
                const uint8_t* const shared = s_q[buffer] + kRowsOf * kRow + (n + 16 * up) * kRopeRow;
                v4f s[kOf];
#pragma unroll
                for (int c = 0; c < kOf; ++c) s[c] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const uint8_t* const at = 4 * i >= kOwn ? shared + ((4 * i - kOwn + h4) ^ ((n >> 1) & 7)) * 16
                                              : mem + (kFour ? h4 * kSteps + i : 4 * i + h4) * 16;
                    const V8 q = __builtin_bit_cast(V8, *(const v4u*)at);
#pragma unroll
                    for (int c = 0; c < kOf; ++c) s[c] = E::mma16(q, k[c][i], s[c]);
                }
                // rows 4 h4 + e in s[..][e]
                const v4f less = *(const v4f*)&s_lse[buffer][16 * up + 4 * h4];
                const bool edge = key0 + 16 * kOf - 1 > (int64_t)f.past + div_page((uint32_t)row0, p.rows_div);  // the first row's last key
                float w[kOf][4];
#pragma unroll
                for (int c = 0; c < kOf; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[c][e] = exp2_of(__builtin_fmaf(s[c][e], p.scale2, -less[e]));
                if (edge) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t pos = (int64_t)f.past + div_page((uint32_t)(row0 + 4 * h4 + e), p.rows_div);
#pragma unroll
                        for (int c = 0; c < kOf; ++c)
                            if (key0 + 16 * c + n > pos) w[c][e] = 0.f;
                    }
                }
#pragma unroll
                for (int c = 0; c < kOf; ++c) sum[c] += (w[c][0] + w[c][1]) + (w[c][2] + w[c][3]);
            }
        };

        float total[kGroups], sum[kGroups];  // sums of sums: an error of few of them, not of all
#pragma unroll
        for (int c = 0; c < kGroups; ++c) total[c] = sum[c] = 0.f;
        __syncthreads();  // all are done with the rows before
        load(rt0, 0);
        store(0);
        __syncthreads();
        if constexpr (kStream) {
            // The share's tiles of this request, in halves: the next half's keys are on their way while one is
            // computed, and page entries before them.
            constexpr int kOf = kGroups / 2;
            const int64_t left = first + f.all() < share1 ? first + f.all() - tile0 : share1 - tile0;
            const int32_t halves = 2 * (int32_t)left;
            done = tile0 + left;
            auto key_of = [&](int32_t x) { return (tile + x / 2) * kTile + wave * (16 * kGroups) + x % 2 * (16 * kOf); };
            V8(&half)[2][kOf][kSteps] = *reinterpret_cast<V8(*)[2][kOf][kSteps]>(&k);
            int32_t at[3][kOf];  // page entries of three halves
            float old[2][kOf];
            auto look = [&](int32_t x, int32_t (&to)[kOf]) {
#pragma unroll
                for (int c = 0; c < kOf; ++c) to[c] = entry_of(key_of(x) + 16 * c + n);
            };
            auto fetch = [&](int32_t x, const int32_t (&entry)[kOf], V8 (&to)[kOf][kSteps], float (&was)[kOf]) {
#pragma unroll
                for (int c = 0; c < kOf; ++c) load_key(to[c], entry[c], key_of(x) + 16 * c + n);
#pragma unroll
                for (int c = 0; c < kOf; ++c) {
                    const int32_t key = key_of(x) + 16 * c + n;
                    was[c] = is_there(entry[c], key) && key < had ? *weight_of(entry[c], key) : 0.f;
                }
            };
            auto turn = [&](auto b, int32_t x) {
                constexpr int kNow = decltype(b)::value;
                if (x + 1 < halves) {
                    // (entries first: a wait for them waits for all loads before them)
                    look(x + 2, at[2]);
                    __builtin_amdgcn_sched_barrier(0);
                    fetch(x + 1, at[1], half[kNow ^ 1], old[kNow ^ 1]);
                }
                float sums[kOf] = {};
                asm volatile("" ::: "memory");  // the queries stay in LDS: registers are for keys on their way
                rows_of(std::integral_constant<int, kOf>{}, half[kNow], key_of(x), 0, 0, sums);
#pragma unroll
                for (int c = 0; c < kOf; ++c) {
                    sums[c] += __shfl_xor(sums[c], 16);
                    sums[c] += __shfl_xor(sums[c], 32);
                    const int32_t key = key_of(x) + 16 * c + n;
                    if (h4 == c && is_there(at[0][c], key)) *weight_of(at[0][c], key) = old[kNow][c] + sums[c];
                    at[0][c] = at[1][c];
                    at[1][c] = at[2][c];
                }
            };
            look(0, at[0]);
            look(1, at[1]);
            fetch(0, at[0], half[0], old[0]);
            for (int32_t x = 0; x < halves; x += 2) {
                turn(std::integral_constant<int, 0>{}, x);
                turn(std::integral_constant<int, 1>{}, x + 1);
            }
        } else {
        for (int32_t rt = rt0; rt < rt1; ++rt) {
            const int buffer = (rt - rt0) & 1;
            if (rt + 1 < rt1) load(rt + 1, buffer ^ 1);
            rows_of(std::integral_constant<int, kGroups>{}, k, k0, rt, buffer, sum);
            if (((rt - rt0) & 31) == 31) {
#pragma unroll
                for (int c = 0; c < kGroups; ++c) {
                    total[c] += sum[c];
                    sum[c] = 0.f;
                }
            }
            if (rt + 1 < rt1) store(buffer ^ 1);
            __syncthreads();
        }
#pragma unroll
        for (int c = 0; c < kGroups; ++c) {
            total[c] += sum[c];
            total[c] += __shfl_xor(total[c], 16);
            total[c] += __shfl_xor(total[c], 32);
        }
        // a quarter of the lanes for each group, in turn
#pragma unroll
        for (int c = 0; c < kGroups; ++c) {
            if (h4 != (c & 3)) continue;
            const int in_tile = (wave * kGroups + c) * 16 + n;
            if (part) {
                to[in_tile] = total[c];
            } else if (is_there(entry[c], tile * kTile + in_tile)) {
                const int32_t key = tile * kTile + in_tile;
                float* const at = weight_of(entry[c], key);
                *at = key < had ? *at + total[c] : total[c];
            }
        }
        }
    }
}

// Requests of one row tile over 16-bit keys: as the other kernel's stream, but K passes through LDS, whole rows a load
// and nothing through registers on its way; each wave has four places for 32 keys and fetches three ahead, and of
// page entries, which places follow from, six. 64 requests of 120 to 8,190 tokens take 93 us; with keys in registers,
// 64-byte pieces a load, 121; without the hint that rows are read once 107.
template <int kDim, bool kHalf>
__global__ __launch_bounds__(kThreads) void k_weigh_stream(WeighPlan p) {
    using E = Elem<kHalf>;
    using V8 = typename E::v8;
    constexpr int kTile = keys_of(0), kSteps = kDim / 32, kColumns = kDim / 8;
    constexpr int kRow = kDim * 2 + 16;                // of a query in LDS, as above
    constexpr int kHalfKeys = 32, kPart = kHalfKeys * kDim * 2;
    constexpr int kLines = 64 / kColumns, kFetches = kHalfKeys / kLines;  // rows of a load, loads of a half
    constexpr int kPlaces = 4, kAhead = kPlaces - 1, kEntries = 2 * kPlaces;
    constexpr int kOps = kFetches + 2;                 // loads of a turn: entries, rows, old weights
    __shared__ __attribute__((aligned(256))) uint8_t s_keys[kWaves][kPlaces][kPart];
    __shared__ int32_t s_entry[kWaves][kEntries][64];
    __shared__ float s_old[kWaves][kPlaces][64];
    __shared__ __attribute__((aligned(16))) uint8_t s_q[kRowsOf * kRow];
    __shared__ __attribute__((aligned(16))) float s_lse[kRowsOf];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, h4 = lane >> 4;
    // (a die's workgroups, every eighth, so read pages of all heads: 106 us and 113 where it had one head)
    const int head = blockIdx.x / p.streams, share = blockIdx.x % p.streams;
    int r;
    int64_t first;
    Items f;
    const Shares shares = find_share<kWaves>(
        p.R, p.streams, [&](int i) { return items_of(p, i, kTile, true); }, share, false, r, f, first);
    if (share >= shares.count) return;
    const int64_t share1 = shares.begin(share + 1);
    for (int64_t done = shares.begin(share); done < share1;) {
        while (done >= first + f.all()) {
            first += f.all();
            f = items_of(p, ++r, kTile, true);
        }
        const int32_t tile = (int32_t)(done - first);
        const int64_t left = first + f.all() < share1 ? first + f.all() - done : share1 - done;
        done += left;
        const int32_t halves = 2 * (int32_t)left;
        const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
        const int32_t end = (int32_t)((int64_t)f.past + f.n < limit ? (int64_t)f.past + f.n : limit);
        const int all_rows = f.n * p.group;
        const int32_t* const table = p.table + (int64_t)r * p.max_blocks;
        const int32_t had = p.weighed ? p.weighed[r] : p.context[r];  // tokens that have weights

        __syncthreads();  // all are done with the rows before
        auto place = [&](int j, int& token, int& sub) {
            const int row = j < all_rows ? j : all_rows - 1;
            token = (int)div_page((uint32_t)row, p.rows_div);
            sub = row - token * p.group;
        };
#pragma unroll
        for (int i = 0; i < kRowsOf * kColumns / kThreads; ++i) {
            const int at = threadIdx.x + i * kThreads, c = at % kColumns, j = at / kColumns;
            int token, sub;
            place(j, token, sub);
            *(v4u*)(s_q + j * kRow + c * 16) =
                *(const v4u*)((const uint8_t*)p.q.p + ((f.begin + token) * p.q.token +
                                                      (int64_t)(head * p.group + sub) * p.q.head) * 2 + c * 16);
        }
        if (threadIdx.x < kRowsOf) {
            int token, sub;
            place(threadIdx.x, token, sub);
            const float lse = (int)threadIdx.x < all_rows
                                  ? p.lse[(f.begin + token) * p.q_heads + head * p.group + sub] : -INFINITY;
            // rows that saw no key, and those that do not exist, give nothing: a weight of 2^-inf
            s_lse[threadIdx.x] = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f;
        }
        __syncthreads();

        // 16-byte columns of a row in LDS are turned, so that 16 lanes which read one of 16 rows find 16 places
        auto turn = [](int row) { return kDim == 128 ? row & 15 : (row >> 1) & 7; };
        auto key_of = [&](int32_t x) { return (tile + x / 2) * kTile + wave * 64 + x % 2 * kHalfKeys; };
        auto look = [&](int32_t x) {  // entries of a half's keys (past the end: the last one's)
            const int32_t key = key_of(x) + (lane & 31);
            fetch4_at(table + div_page((uint32_t)(key < end ? key : end - 1), p.kv.div),
                      lds_of(s_entry[wave][x % kEntries]));
        };
        // a lane's key of a half: whether it is there, and its line of the head and page
        auto find = [&](int32_t x, int32_t& entry, uint32_t& slot) {
            const int32_t key = key_of(x) + (lane & 31);
            entry = s_entry[wave][x % kEntries][lane];
            const bool there = key < end && entry >= 0 && entry < (int32_t)p.kv.blocks;
            entry = there ? entry : 0;
            slot = there ? (uint32_t)key - div_page((uint32_t)key, p.kv.div) * p.kv.div.page : 0u;
            return there;
        };
        auto weight_of = [&](int32_t entry, uint32_t slot) {
            return p.weights + ((int64_t)entry * p.kv.heads + head) * p.kv.div.page + slot;
        };
        auto fetch = [&](int32_t x) {
            int32_t entry;
            uint32_t slot;
            find(x, entry, slot);
            // in units of 16 bytes: a plane is 64 GiB at most
            const uint32_t at = (uint32_t)entry * (p.kv.slab / 16) + ((uint32_t)head * p.kv.div.page + slot) * kColumns;
            const uint32_t to = lds_of(s_keys[wave][x % kPlaces]);
#pragma unroll
            for (int i = 0; i < kFetches; ++i) {
                const int j = i * kLines + lane / kColumns;
                const uint32_t row = (uint32_t)__builtin_amdgcn_ds_bpermute(j * 4, (int)at);
                fetch16_once_at(p.kv.k + ((uint64_t)(row + ((lane % kColumns) ^ turn(j))) << 4), to + i * 1024);
            }
            fetch4_at(weight_of(entry, slot), lds_of(s_old[wave][x % kPlaces]));
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) look(i);
        arrive<0>();
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {  // as in the loop's turns before the first
            look(kAhead + i);
            if (i < halves) fetch(i);
        }
        float held = 0.f;  // an even half's weights: those of two are written at once
        float* held_at = nullptr;
        for (int32_t x = 0; x < halves; ++x) {
            // Left under way: what the two turns before have fetched. Stores may be, too: then this waits for more.
            if (x + kAhead - 1 < halves)
                arrive<(kAhead - 1) * kOps>();
            else
                arrive<0>();
            look(x + 2 * kAhead);
            if (x + kAhead < halves) fetch(x + kAhead);
            V8 k[2][kSteps];
            const uint8_t* const mem = s_keys[wave][x % kPlaces];
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
                    k[c][i] = __builtin_bit_cast(V8, *(const v4u*)(mem + (16 * c + n) * (kDim * 2) +
                                                                  ((4 * i + h4) ^ turn(n)) * 16));
            const int32_t key0 = key_of(x);
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int up = 0; up < 2; ++up) {
                const int row0 = 16 * up;
                if (up && row0 >= all_rows) break;
                v4f s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const V8 q = __builtin_bit_cast(V8, *(const v4u*)(s_q + (n + row0) * kRow + (4 * i + h4) * 16));
#pragma unroll
                    for (int c = 0; c < 2; ++c) s[c] = E::mma16(q, k[c][i], s[c]);
                }
                // rows 4 h4 + e in s[..][e]
                const v4f less = *(const v4f*)&s_lse[row0 + 4 * h4];
                float w[2][4];
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[c][e] = exp2_of(__builtin_fmaf(s[c][e], p.scale2, -less[e]));
                if (key0 + kHalfKeys - 1 > (int64_t)f.past + div_page((uint32_t)row0, p.rows_div)) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t pos = (int64_t)f.past + div_page((uint32_t)(row0 + 4 * h4 + e), p.rows_div);
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            if (key0 + 16 * c + n > pos) w[c][e] = 0.f;
                    }
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) sum[c] += (w[c][0] + w[c][1]) + (w[c][2] + w[c][3]);
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                sum[c] += __shfl_xor(sum[c], 16);
                sum[c] += __shfl_xor(sum[c], 32);
            }
            int32_t entry;
            uint32_t slot;
            const bool there = find(x, entry, slot);
            const float old = key0 + (lane & 31) < had ? s_old[wave][x % kPlaces][lane] : 0.f;
            const float now = old + (h4 & 1 ? sum[1] : sum[0]);
            float* const now_at = there ? weight_of(entry, slot) : nullptr;
            if (x & 1) {
                float* const to = lane < kHalfKeys ? held_at : now_at;
                if (to) *to = lane < kHalfKeys ? held : now;
            }
            held = now;
            held_at = now_at;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the half is read: a later one may overwrite it
        }
        arrive<0>();  // entries that no half uses
    }
}

// The first workgroups take the requests of one row tile, the others those of several: in one launch, since the
// host does not know of which there are any.
template <int kDim, bool kHalf, int kLayout>
__global__ __launch_bounds__(kThreads, weigh_waves(kDim)) void k_weigh(WeighPlan p) {
    __shared__ __attribute__((aligned(16))) uint8_t s_q[2][WeighShape<kDim, kLayout>::kBuffer];
    __shared__ __attribute__((aligned(16))) float s_lse[2][kRowsOf];
    const int first = p.streams * p.kv.heads;
    if ((int)blockIdx.x < first)
        weigh<kDim, kHalf, kLayout, true>(p, blockIdx.x, s_q, s_lse);
    else
        weigh<kDim, kHalf, kLayout, false>(p, blockIdx.x - first, s_q, s_lse);
}

// Adds the parts of tiles that several shares have: the workgroup of the share that begins a tile does.
template <int kLayout>
__global__ __launch_bounds__(keys_of(kLayout)) void k_weigh_join(WeighPlan p) {
    constexpr int kTile = keys_of(kLayout);
    const int head = blockIdx.x % p.kv.heads, share = blockIdx.x / p.kv.heads;
    int r;
    int64_t first;
    Items f;
    const Shares shares = find_share<kTile / 64>(
        p.R, p.shares, [&](int i) { return items_of(p, i, kTile, false); }, share, true, r, f, first);
    if (share >= shares.count || f.rows <= p.whole) return;
    const int64_t share0 = shares.begin(share), share1 = shares.begin(share + 1);
    const int32_t tile = tile_of(f, share1 - 1 - first);
    const int64_t tile0 = first + f.before(tile), tile1 = first + f.before(tile + 1);
    if (tile0 < share0 || tile1 <= share1) return;
    const int64_t last = shares.of(tile1 - 1);
    const int64_t step = 2 * (int64_t)p.kv.heads * kTile;
    const float* from = p.parts + (2 * (int64_t)blockIdx.x + 1) * kTile + threadIdx.x;
    float sum = *from;
    from += step - kTile;  // the first part of the next share
#pragma unroll 8
    for (int64_t i = share + 1; i <= last; ++i, from += step) sum += *from;
    const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
    const int64_t end = (int64_t)f.past + f.n < limit ? (int64_t)f.past + f.n : limit;
    const int64_t key = (int64_t)tile * kTile + threadIdx.x;
    if (key < end) put_weight(p, r, head, (int32_t)key, sum);
}

int32_t shares_of(int32_t heads, int workgroups) { return workgroups > heads ? workgroups / heads : 1; }

template <int kDim, bool kHalf, int kLayout>
hipError_t run(const WeighPlan& plan, hipStream_t s) {
    WeighPlan p = plan;
    const int64_t rows = p.n_tokens * p.group;
    // Single tokens and drafts, by the average request. Items of a tile that is not cut: of these, more, since without
    // cut tiles there is no second kernel (64 tokens 4 us less; 6 prompts of up to 92 tokens by 64 heads 20 us with 4,
    // 34 with 16).
    const bool few = rows <= (int64_t)kRowsOf * p.R;
    p.whole = few ? 16 : 4;
    // As many workgroups of each kind as the device holds. Of a single request the host knows how many row tiles
    // it has at most (rows before and behind it, and those before position 0, are not its), so it has one kind.
    const int32_t shares = shares_of(p.kv.heads, p.cus * weigh_waves(kDim));
    p.apart = p.R > 1 || rows <= kRowsOf;
    p.streams = p.apart ? shares : 0;
    p.shares = rows > kRowsOf ? shares : 0;
    if constexpr (kLayout == 0) {
        // (beside longer requests in a launch of its own, which takes longer than it saves where those are most)
        if (few && p.streams) {
            p.streams = shares_of(p.kv.heads, p.cus);
            hipLaunchKernelGGL((k_weigh_stream<kDim, kHalf>), dim3((unsigned)(p.streams * p.kv.heads)), dim3(kThreads), 0,
                               s, p);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            p.streams = 0;
        }
    }
    if (p.streams + p.shares > 0)
        hipLaunchKernelGGL((k_weigh<kDim, kHalf, kLayout>), dim3((unsigned)((p.streams + p.shares) * p.kv.heads)),
                           dim3(kThreads), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || rows <= p.whole * kRowsOf) return e;  // no request can have a tile that is cut
    hipLaunchKernelGGL((k_weigh_join<kLayout>), dim3((unsigned)(p.shares * p.kv.heads)), dim3(keys_of(kLayout)), 0, s, p);
    return hipGetLastError();
}

template <int kDim>
hipError_t run_kind(const WeighPlan& p, hipStream_t s) {
    if (p.kv.kind == PTSTORE_KV_MXFP4) return run<kDim, false, 1>(p, s);
    return p.kv.kind == PTSTORE_KV_FP16 ? run<kDim, true, 0>(p, s) : run<kDim, false, 0>(p, s);
}

template <int kDim>
hipError_t run_latent(const WeighPlan& p, hipStream_t s) {
    return p.latent.kind == PTSTORE_KV_FP16 ? run<kDim, true, kLatent>(p, s) : run<kDim, false, kLatent>(p, s);
}

}  // namespace

int64_t weigh_workspace(int32_t heads, int cus) {
    return 2ll * shares_of(heads, cus * 3) * heads * keys_of(0) * (int64_t)sizeof(float);
}

hipError_t launch_weigh(const WeighPlan& p, hipStream_t s) {
    if (p.is_latent) return p.latent.latent == 512 ? run_latent<512 + kRope>(p, s) : run_latent<256 + kRope>(p, s);
    return p.kv.dim == 128 ? run_kind<128>(p, s) : run_kind<64>(p, s);
}

}  // namespace ptsd
