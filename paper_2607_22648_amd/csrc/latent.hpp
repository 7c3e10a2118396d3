// Operators of a latent cache: rows in and out of their pages, and attention over them
// (latent_api.hip checks the calls; latent_rows.hip, latent_attend.hip and latent_prompt.hip hold
// the kernels). What they share is here.
//
// One layer is a plane [cache block][slot][latent + rope] of 16-bit values: a token's row is what
// all heads' keys and values come from, then the part of the keys that all heads share.
#pragma once

#include "paged.hpp"

namespace ptsd {

constexpr int kRope = 64;  // values of the shared part of a key

struct LatentPlane {
    uint8_t* rows;
    int64_t blocks;
    int32_t latent;  // 256 or 512
    int32_t kind;    // PTSTORE_KV_BF16, PTSTORE_KV_FP16
    PageDiv div;
    uint32_t line;   // a row, in units of 16 bytes: a plane's rows are numbered in 32 bits of them
};

struct LatentPlan {
    LatentPlane kv;
    Rows ql, qr;  // queries: the latent part, the shared part
    Rows out;
    float* lse;
    const int64_t* offsets;
    const int32_t* context;
    const int32_t* table;
    int64_t n_tokens;
    int32_t R, max_blocks;
    int32_t group;     // rows of a token: all heads
    int32_t few_rows;  // no limit here
    float scale2;      // scale * log2(e): scores in base 2
    float* parts;      // workspace
    int32_t shares;
};

constexpr int kNope = 128, kValue = 128;  // of a head: values of a key's own part, of a value

// The expanded form: keys and values of all heads, packed [head][key], in the workspace.
struct ExpandedPlan {
    LatentPlane kv;
    Rows qn, qr, out;  // queries: a head's own part, the shared part
    Rows wk, wv;       // [head][row of the head][latent]: `token` is the row's stride
    float* lse;
    const int64_t* offsets;
    const int32_t* context;
    const int32_t* table;
    const int64_t* key_offsets;
    int64_t n_tokens, n_keys;
    int32_t R, max_blocks, heads;
    int32_t group, few_rows;  // rows of a token: one a head; no limit
    float scale2;
    uint8_t *k, *v;   // [head][key]: 128 nearest 16-bit values, 128 of what is left
    uint8_t* rope;    // [key][64]
    int32_t* there;   // [key] whether its page exists
    int32_t parts;    // of the heads, each with dies of its own
};

int64_t expanded_workspace(int32_t heads, int64_t n_keys);  // bytes
void place_expanded(ExpandedPlan* p, void* workspace);
hipError_t launch_expanded(const ExpandedPlan& p, int cus, hipStream_t s);

const char* plane_of(const ptstore_latent_t* cache, LatentPlane* out);  // or why not
const char* batch_of(int64_t n_tokens, int32_t R, int32_t max_blocks, int32_t block_tokens, int32_t heads);
hipError_t launch_latent_append(const LatentPlane& kv, const void* latent, int64_t latent_stride, const void* rope,
                                int64_t rope_stride, const int64_t* slots, int64_t n, hipStream_t s);
hipError_t launch_latent_read(const LatentPlane& kv, void* latent, int64_t latent_stride, void* rope,
                              int64_t rope_stride, const int64_t* slots, int64_t n, hipStream_t s);
int64_t latent_workspace(int latent, int cus);  // bytes
hipError_t launch_latent(const LatentPlan& p, hipStream_t s);

}  // namespace ptsd
