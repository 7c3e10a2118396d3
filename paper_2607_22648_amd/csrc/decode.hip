// Attention of few query rows a KV head: single tokens, and the few of a draft
// that is checked.
//
// Bound by memory: a request's K and V are read once and every other byte is
// small beside them. What matters is that all compute units read all the time,
// whatever the lengths. So the batch's work, in steps of keys, is laid out end to end
// (request, tile of query rows, KV head, step) and cut into equal shares, one
// for each workgroup that the device holds at once. A share that ends inside a
// (tile, KV head) leaves its maximum, sum and output in the workspace, two such
// parts a workgroup at most, and a second kernel joins them. Workgroups for fixed
// parts of a request were up to 1.3 times slower by how their number fell on the
// device, and paid their start per part. The KV heads of a share run side by side, so
// that neighbouring slabs are read together (217 us instead of 194 otherwise, 64
// requests of 120 to 8,190 keys).
//
// A workgroup is four waves that share nothing until a (tile, KV head) is done: wave
// w takes every fourth piece of a share's keys. 16-bit K and V rows are loaded whole
// (four rows of 256 bytes an instruction; in 64-byte pieces, as the matrix
// instruction takes K, they reached 5.8 TB/s instead of 6.4), pass through 8 KiB of LDS
// that only this wave uses, and are read as the matrix instructions want them, V
// transposed. 4-bit K is loaded in that order from the start: its rows are 64
// bytes. The next piece's loads are issued as soon as a register is free, so that each
// wave keeps a piece's bytes in flight while it computes.
//
// 8 KV heads of 128 with 4 query heads each, one token a request (without the join,
// 5 us): 64 requests of 8,192 keys 315 us, 6.8 TB/s of the 7.2 that a plain read reaches;
// of 4-bit keys 97 us, 5.9 TB/s, where widening the codes (a quarter of the
// instructions) and the two exchanges of a row's exponent take as long as the memory.
// One request of 778 keys takes 7.7 us, about what a chain of its trips through
// memory (lengths, page, K, V) takes.
//
// Query rows are the (token, head of the group) pairs of one KV head, 16 to a
// tile: with 4 heads to a KV head a single token fills 4 of the 16 columns, and
// the matrix instructions idle for the rest, which costs nothing here.
#include "attend.hpp"
#include "shares.hpp"

namespace ptsd {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;

// Keys of a step: a piece for each wave.
constexpr int step_keys(bool four) { return kWaves * (four ? 64 : 32); }

// Floats of a part in the workspace: rows, then each one's maximum and sum.
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
// bits. Rows of 128 bytes (dim 64) already differ by parity. The lowest bit is free,
// since a read takes both columns of a pair: 4-bit rows, whose lanes write columns 2
// or 4 apart, turn by it too.
template <int D, bool kFour>
__device__ inline int turn_v(int row) {
    const int low = kFour ? (row >> 1) & 1 : 0;
    if constexpr (D == 128)
        return 2 * ((row & 3) + 4 * ((row >> 3) & 1)) + low;
    else
        return 2 * (((row >> 1) & 1) + 2 * ((row >> 3) & 1)) + low;
}

template <int D, bool kHalf, bool kFour>
__global__ __launch_bounds__(kThreads, 2) void k_decode(AttendPlan p) {
    using E = Elem<kHalf>;
    constexpr int kKeys = kFour ? 64 : 32;        // keys of a wave's piece
    constexpr int kStepKeys = step_keys(kFour);
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

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, h4 = lane >> 4;  // query column, quarter
    const int64_t limit = (int64_t)p.max_blocks * p.kv.div.page;
    const int head = blockIdx.x % p.kv.heads, share = blockIdx.x / p.kv.heads;
    int r;
    int64_t first;  // the request's first step
    Work f;
    const Shares shares = find_step<kDecodeRows, kWaves>(p, kStepKeys, share, false, r, f, first);
    if (share >= shares.count) return;
    const int64_t share0 = shares.begin(share), share1 = shares.begin(share + 1);
    for (int64_t done = share0; done < share1;) {
    while (done >= first + f.all()) {  // on to the next request with work
        first += f.all();
        f = work_of<kDecodeRows>(p, ++r, kStepKeys);
    }
    const int tile = (int)((done - first) / f.steps);
    const int64_t tile0 = first + (int64_t)tile * f.steps;  // the tile's first step
    const int step0 = (int)(done - tile0);
    const int step1 = share1 - tile0 < f.steps ? (int)(share1 - tile0) : f.steps;
    done = tile0 + step1;

    // the tile's rows see keys up to `end`; those of this share are [k0, k1)
    const int rows_left = f.n * p.group - tile * kDecodeRows;
    const int rows = rows_left < kDecodeRows ? rows_left : kDecodeRows;
    const int row = tile * kDecodeRows + (n < rows ? n : rows - 1);
    const int token = row / p.group, sub = row - token * p.group;
    int64_t seen = f.past + (tile * kDecodeRows + rows - 1) / p.group + 1;
    seen = seen < 0 ? 0 : (seen > limit ? limit : seen);
    const int32_t end = (int32_t)seen;
    const int32_t k0 = step0 * kStepKeys;
    const int32_t k1 = end - k0 < (step1 - step0) * kStepKeys ? end : step1 * kStepKeys;
    const int64_t pos64 = f.past + token;  // the last key this lane's query sees
    const int32_t pos = pos64 < limit ? (int32_t)pos64 : (int32_t)limit;
    const int64_t first64 = f.past + tile * kDecodeRows / p.group;
    const int32_t all_see = first64 < limit ? (int32_t)first64 : (int32_t)limit;

    const int32_t* table = p.table + (int64_t)r * p.max_blocks;
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
    __builtin_amdgcn_sched_barrier(0);

    v4f o[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i] = v4f{0, 0, 0, 0};
    float top = kLowest, sum = 0.f;
    bool far = false;  // scores are scaled before the maximum is taken

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
    auto four = [&](const uint8_t* at) {
        if constexpr (D == 128) return once16(at);
        const v2u x = once8(at);
        return v4u{x[0], x[1], 0u, 0u};
    };
    auto load_k = [&](const KeyRow& r) {
        if constexpr (kFour) {
            kpow = load_powers<D>(p.kv.k, r.power);
            uint32_t at[kGroups];
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
                at[g] = (uint32_t)__shfl((int)r.at, 32 * (g >> 1) + 4 * (g & 1) + key_of_row);
            together(at);
#pragma unroll
            for (int g = 0; g < kGroups; ++g) kreg[g] = four(kbase + ((uint64_t)at[g] << 4));
        } else {
            uint32_t at[kPieces];
#pragma unroll
            for (int i = 0; i < kPieces; ++i) at[i] = (uint32_t)__shfl((int)r.at, i * (64 / kLanes) + lane / kLanes);
            together(at);
#pragma unroll
            for (int i = 0; i < kPieces; ++i) kreg[i] = once16(kbase + ((uint64_t)at[i] << 4));
        }
    };
    auto load_v = [&](const KeyRow& r) {
        constexpr int kLoads = kFour ? kKeys / kVKeys : kPieces;
        if constexpr (kFour) vpow = load_powers<D>(p.kv.v, r.power);
        uint32_t at[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            at[i] = (uint32_t)__shfl((int)r.at, kFour ? i * kVKeys + (lane >> 2) : i * (64 / kLanes) + lane / kLanes);
        together(at);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint8_t* row = vbase + ((uint64_t)at[i] << 4);
            if constexpr (kFour)
                vreg[i] = four(row);
            else
                vreg[i] = once16(row);
        }
    };
    // the exponent of the lane's quarter q of a row, from the word of the row's
    auto power = [&](uint32_t word, int quarter) { return (word >> (quarter * (D / 4) / kGroup * 8)) & 255u; };

    // The order of loads is fixed, since a wait for one waits for all before it: the
    // queries; then, for each piece, the page entries of the piece after it, its K, its V.
    // None depends on a branch, past which a wait would have to allow for either
    // way: what lies past the share's end reads block 0.
    int32_t at = k0 + wave * kKeys;
    bool there;
    int32_t entry = page_entry(p, table, at + step_key, k1);
    KeyRow place = key_row<D, kFour>(p.kv, entry, at + step_key, k1, head_row, there);
    uint64_t valid = __ballot(there);
    entry = page_entry(p, table, at + stride + step_key, k1);
    __builtin_amdgcn_sched_barrier(0);
    load_k(place);
    __builtin_amdgcn_sched_barrier(0);
    load_v(place);
    __builtin_amdgcn_sched_barrier(0);
    uint8_t* const lds = s_mem.v[wave];
    bool endless = false;  // a V value that is not finite lies behind the first row's last key

    while (at < k1) {
        // 16-bit: LDS addresses are formed anew each time; kept, they take two dozen
        // registers
        int here = lane;
        if constexpr (!kFour) asm volatile("" : "+v"(here));
        // scores of column n: keys 32 b + 8 h4 + 4 (g & 1) + i in s[g][i], b = g >> 1
        v4f s[kGroups];
        if constexpr (!kFour) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int key = i * (64 / kLanes) + here / kLanes;
                *(v4u*)(lds + key * kRow + (((here % kLanes) ^ turn_k<D>(key)) * 16)) = kreg[i];
            }
            wave_order();
        }
        float kstep[kFour ? kGroups : 1];
        if constexpr (kFour) {
            uint32_t word[kGroups];
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
                word[g] = (uint32_t)__shfl((int)kpow, 32 * (g >> 1) + 4 * (g & 1) + key_of_row);
            together(word);
#pragma unroll
            for (int g = 0; g < kGroups; ++g) kstep[g] = step_of(power(word[g], h4));
        }
        const int krow = 8 * ((here & 15) >> 2) + (here & 3);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) s[g] = v4f{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < kSteps; ++t)
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int key = 4 * (g & 1) + krow;
                v4u a;
                if constexpr (kFour)
                    a = widen8(kreg[g][t], kstep[g]);
                else
                    a = *(const v4u*)(lds + key * kRow + (((4 * t + (here >> 4)) ^ turn_k<D>(key)) * 16));
                s[g] = E::mma16(__builtin_bit_cast(typename E::v8, a), __builtin_bit_cast(typename E::v8, q[t]), s[g]);
            }
        wave_order();
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
        auto scale_now = [&] {
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[g][i] = product(s[g][i], p.scale2);
            most = product(most, p.scale2);
        };
        if (far) scale_now();
        float top2 = fmaxf(top, __builtin_fmaf(most, far ? 1.f : p.scale2, E::kRoom));
        if (__any(top2 > top)) {
            if (!far && __any(is_far(top2))) {
                far = true;
                scale_now();
                top2 = fmaxf(top, most + E::kRoom);
            }
            const float less = exp2_of(top - top2);
            sum *= less;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[i] *= less;
            top = top2;
        }
        const float scale = far ? 1.f : p.scale2;
        v4u w[kKeys / 32];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[g][i] = exp2_of(__builtin_fmaf(s[g][i], scale, -top));
                sum += s[g][i];
            }
            // Weights enter the second product as 16-bit values, as V does; the sum takes them
            // as they are. Each is off by half a step of the type at most, as much as the
            // output's own rounding adds; over many keys the errors average out, and the largest
            // weight of a row, a power of two, has next to none.
            w[g >> 1][2 * (g & 1)] = pack2<kHalf>(s[g][0], s[g][1]);
            w[g >> 1][2 * (g & 1) + 1] = pack2<kHalf>(s[g][2], s[g][3]);
        }

        uint32_t vword[kFour ? kKeys / kVKeys : 1];
        if constexpr (kFour) {
#pragma unroll
            for (int j = 0; j < kKeys / kVKeys; ++j) vword[j] = (uint32_t)__shfl((int)vpow, j * kVKeys + (here >> 2));
            together(vword);
        }
#pragma unroll
        for (int b = 0; b < kKeys / 32; ++b) {
            // V's rows of 32 keys into LDS
            if constexpr (kFour) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int key = i * kVKeys + (here >> 2), j = 2 * b + i;
                    const float step = step_of(power(vword[j], here & 3));
#pragma unroll
                    for (int c = 0; c < kWords; ++c) {
                        const int col = (here & 3) * kWords + c;
                        *(v4u*)(lds + key * kRow + ((col ^ turn_v<D, kFour>(key)) * 16)) = widen8(vreg[j][c], step);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int key = i * (64 / kLanes) + here / kLanes;
                    *(v4u*)(lds + key * kRow + (((here % kLanes) ^ turn_v<D, kFour>(key)) * 16)) = vreg[i];
                }
            }
            wave_order();
            if (b == kKeys / 32 - 1) {
                __builtin_amdgcn_sched_barrier(0);
                load_v(place);
                __builtin_amdgcn_sched_barrier(0);
            }
            // column d of 32 keys, 8 of them a lane: two transposed reads
            const int m = here & 15, vrow = 8 * (here >> 4) + (m >> 2);
            v4u vt[D / 16];
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const int col = 2 * i + ((m & 3) >> 1), in = (m & 1) * 8;
                const v2u lo = read_transposed(lds + vrow * kRow + ((col ^ turn_v<D, kFour>(vrow)) * 16) + in);
                const v2u hi = read_transposed(lds + (vrow + 4) * kRow + ((col ^ turn_v<D, kFour>(vrow + 4)) * 16) + in);
                vt[i] = join(lo, hi);
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                o[i] = E::mma16(__builtin_bit_cast(typename E::v8, vt[i]),
                                __builtin_bit_cast(typename E::v8, w[b]), o[i]);
            wave_order();
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
    if (orow < rows) {
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
        if (step0 > 0 || step1 < f.steps) {
            // a part: of a tile that began in an earlier share, or one that goes on
            float* to = p.parts + (2 * (int64_t)blockIdx.x + (step0 > 0 ? 0 : 1)) * part_floats(D);
            *(v4f*)(to + orow * D + oc * 8) = v4f{acc[0], acc[1], acc[2], acc[3]};
            *(v4f*)(to + orow * D + oc * 8 + 4) = v4f{acc[4], acc[5], acc[6], acc[7]};
            if (oc == 0) *(v2f*)(to + kDecodeRows * D + 2 * orow) = v2f{all, total};
        } else {
            const int out_row = tile * kDecodeRows + orow;
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
    }
    __syncthreads();  // the next tile writes there
    }
}

// A row's parts so far: 4 dimensions of the output, the maximum, the sum.
struct Joined {
    v4f acc = {0, 0, 0, 0};
    float all = kLowest, total = 0.f;
    // To a maximum of at least `top`. Sums that then weigh nothing stay in as zeros, and as NaN
    // where they are not finite: a part whose scores are all NaN has the lowest maximum.
    __device__ void raise(float top) {
        const float to = fmaxf(all, top), less = exp2_of(all - to);
        total *= less;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= less;
        all = to;
    }
    // a part whose maximum is not above `all`
    __device__ void add(v4f o, float top, float sum) {
        const float part_of = exp2_of(top - all);
        total += part_of * sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += part_of * o[e];
    }
};

// Joins the parts of a tile that several shares have. The workgroups of all these
// shares but the last take the tile's rows in turn; a workgroup's waves, and each wave's
// halves (dim 64: quarters), divide a row's parts, 4 dimensions a lane, several parts in
// flight, so that 64 parts of a row are one trip to memory. (A kernel of its own:
// joined by the workgroup that writes the last part, which has to pass the parts
// through memory that all dies see, one request of 32,768 keys took 45 us, not 34.)
constexpr int kJoinWaves = 8;

template <int D, bool kHalf, bool kFour>
__global__ __launch_bounds__(kJoinWaves * 64) void k_join(AttendPlan p) {
    constexpr int kRowLanes = D / 4, kPhases = 64 / kRowLanes, kFlight = 8;
    __shared__ v4f s_acc[kJoinWaves][kRowLanes];
    __shared__ float s_all[kJoinWaves], s_total[kJoinWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int phase = lane / kRowLanes, c = lane % kRowLanes;
    const int head = blockIdx.x % p.kv.heads, share = blockIdx.x / p.kv.heads;
    int r;
    int64_t first;
    Work f;
    const Shares shares = find_step<kDecodeRows, kJoinWaves>(p, step_keys(kFour), share, true, r, f, first);
    if (share >= shares.count) return;
    const int64_t share1 = shares.begin(share + 1);
    const int tile = (int)((share1 - 1 - first) / f.steps);
    const int64_t tile0 = first + (int64_t)tile * f.steps, tile1 = tile0 + f.steps;
    if (tile1 <= share1) return;
    const int share0 = (int)shares.of(tile0);  // the tile's first
    const int parts = (int)(shares.of(tile1 - 1) - share0 + 1);
    const int rows_left = f.n * p.group - tile * kDecodeRows;
    const int rows = rows_left < kDecodeRows ? rows_left : kDecodeRows;
    // rows row0, row0 + parts - 1, ... are this workgroup's
    const int row0 = share - share0;
    if (row0 >= rows) return;
    const int mine = (rows - row0 + parts - 2) / (parts - 1);
    // waves a row: as many as there are, and its parts keep busy
    int slices = mine == 1 ? 8 : mine == 2 ? 4 : mine <= 4 ? 2 : 1;
    while (slices > 1 && slices / 2 * kPhases * kFlight >= parts) slices /= 2;
    const int slice = wave % slices;
    // the first share's second part, then the first of each following
    const float* from = p.parts + (2 * ((int64_t)share0 * p.kv.heads + head) + 1) * part_floats(D);
    const int64_t next = 2ll * p.kv.heads * part_floats(D);
    auto part_at = [&](int i) { return from + i * next - (i > 0 ? part_floats(D) : 0); };
    for (int at = 0; at < mine; at += kJoinWaves / slices) {
        const int row = row0 + (at + wave / slices) * (parts - 1);
        Joined sum;
        for (int i0 = slice * kPhases + phase; i0 < parts && row < rows; i0 += slices * kPhases * kFlight) {
            v4f o[kFlight];
            v2f ms[kFlight];
            float top = kLowest;
#pragma unroll
            for (int u = 0; u < kFlight; ++u) {
                const int i = i0 + u * slices * kPhases;
                const float* part = part_at(i < parts ? i : i0);
                o[u] = *(const v4f*)(part + row * D + c * 4);
                ms[u] = *(const v2f*)(part + kDecodeRows * D + 2 * row);
                if (i >= parts) {
                    o[u] = v4f{0, 0, 0, 0};
                    ms[u] = v2f{-INFINITY, 0.f};
                }
            }
#pragma unroll
            for (int u = 0; u < kFlight; ++u) top = fmaxf(top, ms[u][0]);
            sum.raise(top);
#pragma unroll
            for (int u = 0; u < kFlight; ++u) sum.add(o[u], ms[u][0], ms[u][1]);
        }
        for (int d = kRowLanes; d < 64; d <<= 1) {
            v4f o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = __shfl_xor(sum.acc[e], d);
            const float top = __shfl_xor(sum.all, d), total = __shfl_xor(sum.total, d);
            sum.raise(top);
            sum.add(o, top, total);
        }
        if (slices > 1) {
            __syncthreads();
            if (phase == 0) s_acc[wave][c] = sum.acc;
            if (lane == 0) {
                s_all[wave] = sum.all;
                s_total[wave] = sum.total;
            }
            __syncthreads();
            if (slice == 0)
                for (int u = 1; u < slices; ++u) {
                    sum.raise(s_all[wave + u]);
                    sum.add(s_acc[wave + u][c], s_all[wave + u], s_total[wave + u]);
                }
        }
        if (slice || phase || row >= rows) continue;
        const int out_row = tile * kDecodeRows + row;
        const int ot = out_row / p.group, os = out_row - ot * p.group;
        const int64_t oh = (int64_t)head * p.group + os;
        const float total = sum.total, inv = total != 0.f ? 1.f / total : 0.f;
        const v2u x = {pack2<kHalf>(sum.acc[0] * inv, sum.acc[1] * inv),
                       pack2<kHalf>(sum.acc[2] * inv, sum.acc[3] * inv)};
        *(v2u*)((uint8_t*)p.out.p + ((f.begin + ot) * p.out.token + oh * p.out.head + c * 4) * 2) = x;
        if (p.lse && c == 0)
            p.lse[(f.begin + ot) * p.q_heads + oh] =
                total != 0.f ? (sum.all + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
    }
}

template <int D, bool kHalf, bool kFour>
hipError_t run(const AttendPlan& p, hipStream_t s) {
    const dim3 grid((unsigned)(p.shares * p.kv.heads));
    hipLaunchKernelGGL((k_decode<D, kHalf, kFour>), grid, dim3(kThreads), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_join<D, kHalf, kFour>), grid, dim3(kJoinWaves * 64), 0, s, p);
    return hipGetLastError();
}

template <int D>
hipError_t run_kind(const AttendPlan& p, hipStream_t s) {
    if (p.kv.kind == PTSTORE_KV_MXFP4) return run<D, false, true>(p, s);
    return p.kv.kind == PTSTORE_KV_FP16 ? run<D, true, false>(p, s) : run<D, false, false>(p, s);
}

}  // namespace

// As many as fill the device: two workgroups a compute unit. More, smaller ones even
// out no better and pay their start: 64 requests of 8,192 keys took 4 % longer with
// four a compute unit, 7 % with eight.
int decode_shares(const Planes& kv, int cus) {
    const int shares = 2 * cus / kv.heads;
    return shares > 0 ? shares : 1;
}

int64_t decode_workspace(const Planes& kv, int shares) {
    return 2ll * shares * kv.heads * part_floats(kv.dim) * (int64_t)sizeof(float);
}

hipError_t launch_decode(const AttendPlan& p, hipStream_t s) {
    return p.kv.dim == 128 ? run_kind<128>(p, s) : run_kind<64>(p, s);
}

}  // namespace ptsd
