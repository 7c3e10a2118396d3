// Operators on the weights that attention gave to cached tokens (weight_api.hip checks the calls;
// weigh.hip and keep.hip hold the kernels).
#pragma once

#include "latent.hpp"
#include "paged.hpp"

namespace ptsd {

struct WeighPlan {
    Planes kv;           // the keys, or
    LatentPlane latent;  // a latent cache's (kv.heads is 1, kv.div and kv.blocks its own)
    bool is_latent;
    Rows q, qr;          // queries; a latent cache's shared part of them
    const float* lse;
    const int64_t* offsets;
    const int32_t* context;
    const int32_t* weighed;
    const int32_t* table;
    int64_t n_tokens;
    int32_t R, max_blocks, q_heads, group;
    float scale2;    // scale * log2(e)
    float* weights;  // [block][KV head][slot]
    float* parts;    // workspace
    int32_t streams, shares;  // of requests of one tile of query rows, of the others
    bool apart;               // requests of one tile have workgroups of their own
    int32_t cus, whole;       // compute units; items of a tile that is not cut
    PageDiv rows_div;         // by group
};

int64_t weigh_workspace(int32_t heads, int cus);  // bytes
hipError_t launch_weigh(const WeighPlan& p, hipStream_t s);

struct KeepPlan {
    uint8_t *k, *v;      // the first layer's planes (v null: one plane)
    int64_t layer;       // bytes from a layer's planes to the next one's
    int64_t blocks;
    int32_t layers, heads, R, max_blocks;
    PageDiv div;
    int64_t slab;        // bytes of a block in a plane
    PageDiv slab_rows;   // division by a block's rows
    int32_t row;         // bytes of a row of values or codes, a multiple of 16
    int32_t power;       // bytes of a row's exponents: 0, 2 or 4
    int64_t powers;      // offset of a slab's exponents
    float* weights;      // [layer][block][head][slot]
    const int32_t* context;
    const int32_t* keep;
    int32_t* context_out;
    const int32_t* from;
    const int32_t* to;
    int32_t max_keep, recent;
    int32_t* source;     // workspace: [unit][max_keep] positions that stay
};

int64_t keep_workgroups(const KeepPlan& p);  // at least, of the larger launch
hipError_t launch_keep(const KeepPlan& p, int cus, hipStream_t s);

}  // namespace ptsd
