// Operators of the caller's paged cache: block tables, appends and attention
// (paged_api.hip checks the calls; tables.hip, append.hip, decode.hip and
// prompt.hip hold the kernels). What the kernels share is here.
//
// One layer of a paged cache is a K plane and a V plane, each
// [cache block][slab]. A 16-bit slab is [head][slot][dim]. A 4-bit slab is
// [head][slot][dim/2] codes, then [head][slot][dim/32] exponents, padded to 16
// bytes: every row of codes keeps a power-of-two alignment at any block size,
// which exponents between the rows would break.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ptstore.h"

namespace ptsd {

constexpr int kGroup = 32;          // elements that share one exponent
constexpr uint32_t kEndless = 253;  // exponent bytes from here on read as NaN
constexpr int64_t kMaxCacheBlocks = 1ll << 30;
constexpr int64_t kMaxPlane = 1ll << 36;  // bytes: rows are numbered in 16 bytes, 32 bits

// Division of a key's position (below 2^31) by the page size (or of another such
// number by a constant of the call): with 2^s >=
// 2^31 d and M = ceil(2^s / d), the error M d - 2^s is below d, so n M / 2^s
// rounds down to n / d for every n < 2^31.
struct PageDiv {
    uint32_t mul, shift, page;
};

inline PageDiv page_div(int page) {
    uint32_t s = 31;
    while ((1ull << (s - 31)) < (uint64_t)page) ++s;
    return {(uint32_t)(((1ull << s) + page - 1) / page), s, (uint32_t)page};
}

__device__ inline uint32_t div_page(uint32_t n, const PageDiv& d) {
    return (uint32_t)(((uint64_t)n * d.mul) >> d.shift);
}

struct Planes {
    uint8_t* k;
    uint8_t* v;
    int64_t blocks;
    int32_t heads, dim;
    PageDiv div;
    uint32_t slab;       // bytes of a block's slab
    uint32_t exponents;  // offset of a 4-bit slab's exponents
    int32_t kind;        // PTSTORE_KV_*
};

// Rows of a packed [token][head][dim] tensor: strides in elements.
struct Rows {
    const void* p;
    int64_t token, head;
};

struct TablesPlan {
    const int64_t* offsets;
    int64_t n_tokens;
    const int32_t* context;
    const int32_t* held;
    int32_t R, max_blocks;
    PageDiv div;
    const int32_t* free_blocks;
    int64_t n_free;
    const int64_t* first;
    int32_t* table;
    int64_t* slots;
    int32_t* positions;
    int32_t* held_out;
    int64_t* next;
};

struct AttendPlan {
    Planes kv;
    Rows q, out;
    float* lse;
    const int64_t* offsets;
    const int32_t* context;
    const int32_t* table;
    int64_t n_tokens;
    int32_t R, max_blocks, q_heads, group;  // group: query heads of a KV head
    float scale2;                           // scale * log2(e): scores in base 2
    int32_t few_rows;                       // requests of up to this many rows are decode.hip's alone,
                                            // the others prompt.hip's (0: all are prompt.hip's)
    float* parts;                           // workspace
    int32_t shares;                         // decode.hip: of the batch's work
    int32_t whole, rest, splits;            // prompt.hip: (tile, KV head) pairs done whole, and in parts
};

// Rows a request that decode.hip takes in a batch that both kernels share.
constexpr int kFewRows = 32;

// Query rows of a decode tile (one matrix instruction's columns) and of a
// prompt tile.
constexpr int kDecodeRows = 16;
constexpr int kPromptRows = 128;

// A request's rows are its (token, head of the group) pairs, token first; its
// tiles are numbered from offsets * group / rows + r, which leaves room for
// every request's last, partly filled tile without a prefix sum over the
// batch. Numbers that no request's rows reach have no work.
inline int64_t tile_bound(int64_t n_tokens, int32_t group, int32_t R, int rows) {
    return n_tokens * group / rows + R;
}

const char* planes_of(const ptstore_kv_t* kv, Planes* out);  // or why not
hipError_t launch_tables(const TablesPlan& p, hipStream_t s);
hipError_t launch_append(const Planes& kv, const Rows& k, const Rows& v, const int64_t* slots, int64_t n,
                         hipStream_t s);
hipError_t launch_read(const Planes& kv, const Rows& k, const Rows& v, const int64_t* slots, int64_t n,
                       hipStream_t s);
int decode_shares(const Planes& kv, int cus);
int64_t decode_workspace(const Planes& kv, int shares);  // bytes
hipError_t launch_decode(const AttendPlan& p, hipStream_t s);
void split_prompt(AttendPlan* p, int cus);
int64_t prompt_workspace(const Planes& kv, int cus);  // bytes
hipError_t launch_prompt(const AttendPlan& p, hipStream_t s);

}  // namespace ptsd
