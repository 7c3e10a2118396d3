// The C calls of latent caches (include/ptstore.h): checks on the host, launch rules, no allocation and no
// state.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "checks.hpp"
#include "latent.hpp"
#include "ptstore.h"

namespace ptsd {

const char* plane_of(const ptstore_latent_t* c, LatentPlane* out) {
    if (!c) return "null cache";
    if ((c->kind != PTSTORE_KV_BF16 && c->kind != PTSTORE_KV_FP16) || (c->latent_dim != 256 && c->latent_dim != 512) ||
        c->rope_dim != kRope || c->block_tokens < 1 || c->block_tokens > 64)
        return "the cache's kind (bf16, fp16), latent_dim (256, 512), rope_dim (64) or block_tokens (1..64) is not "
               "supported";
    const int64_t row = 2ll * (c->latent_dim + c->rope_dim);
    if (c->cache_blocks < 0 || c->cache_blocks > kMaxCacheBlocks) return "cache_blocks out of range (0..2^30)";
    if (c->cache_blocks * c->block_tokens * row > kMaxPlane) return "a plane of the cache exceeds 64 GiB";
    if (c->cache_blocks > 0 && (!c->rows || !aligned16(c->rows))) return "the cache's plane must be 16-byte aligned";
    out->rows = static_cast<uint8_t*>(c->rows);
    out->blocks = c->cache_blocks;
    out->latent = c->latent_dim;
    out->kind = c->kind;
    out->div = page_div(c->block_tokens);
    out->line = (uint32_t)(row / 16);
    return nullptr;
}

// The sizes of a batch of `heads` query rows a token.
const char* batch_of(int64_t n_tokens, int32_t R, int32_t max_blocks, int32_t block_tokens, int32_t heads) {
    if (heads < 1) return "heads must be positive";
    if (R < 0 || max_blocks < 1 || (int64_t)R * max_blocks > kMaxEntries || n_tokens < 0 || (R == 0 && n_tokens > 0))
        return "R, max_blocks or n_tokens out of range";
    if ((int64_t)max_blocks * block_tokens > kMaxKeys) return "max_blocks * block_tokens exceeds 2^30";
    // rows are numbered in 32 bits, up to the end of a last tile
    constexpr int64_t most = (1ll << 31) - 128;
    if (n_tokens > most || n_tokens * heads > most) return "n_tokens * heads exceeds 2^31 - 128";
    return nullptr;
}

}  // namespace ptsd

using namespace ptsd;

namespace {

constexpr int64_t kMostKeys = (1ll << 31) - 256;       // of a call's expanded keys: numbered in 31 bits
constexpr int64_t kMaxUnits = kMaxItems / 256 - 8192;  // workgroups of latent_prompt.hip

int move_rows(const char* call, const ptstore_latent_t* cache, const void* latent, int64_t latent_stride,
              const void* rope, int64_t rope_stride, const int64_t* slots, int64_t n, bool read, void* stream) {
    LatentPlane kv;
    if (const char* bad = plane_of(cache, &kv)) return refuse_as(call, bad);
    // pieces of 8 values are numbered in 31 bits
    if (n < 0 || n > (1ll << 31) / kv.line) return refuse_as(call, "n_tokens * (latent_dim + rope_dim) exceeds 2^34");
    if (n == 0) return PTSTORE_OK;
    if (!slots || !rows_ok(latent, latent_stride, 0) || !rows_ok(rope, rope_stride, 0))
        return refuse_as(call, "null argument, or rows of latent or rope not 16-byte aligned");
    const hipError_t e =
        read ? launch_latent_read(kv, const_cast<void*>(latent), latent_stride, const_cast<void*>(rope), rope_stride,
                                  slots, n, (hipStream_t)stream)
             : launch_latent_append(kv, latent, latent_stride, rope, rope_stride, slots, n, (hipStream_t)stream);
    return e == hipSuccess ? PTSTORE_OK : set_last_error(PTSTORE_ERR_HIP, call);
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int ptstore_latent_append(const ptstore_latent_t* cache, const void* latent, int64_t latent_stride, const void* rope,
                          int64_t rope_stride, const int64_t* slots, int64_t n_tokens, void* stream) {
    return move_rows("ptstore_latent_append", cache, latent, latent_stride, rope, rope_stride, slots, n_tokens, false,
                     stream);
}

int ptstore_latent_read(const ptstore_latent_t* cache, void* latent, int64_t latent_stride, void* rope,
                        int64_t rope_stride, const int64_t* slots, int64_t n_tokens, void* stream) {
    return move_rows("ptstore_latent_read", cache, latent, latent_stride, rope, rope_stride, slots, n_tokens, true,
                     stream);
}

int ptstore_latent_attention_workspace(const ptstore_latent_t* cache, int64_t* bytes) {
    LatentPlane kv;
    if (!bytes) return refuse("ptstore_latent_attention_workspace: null argument");
    if (const char* bad = plane_of(cache, &kv)) return refuse_as("ptstore_latent_attention_workspace", bad);
    int cus = 0;
    if (const int rc = compute_units("ptstore_latent_attention_workspace", &cus)) return rc;
    *bytes = latent_workspace(kv.latent, cus);
    return PTSTORE_OK;
}

int ptstore_latent_attention(const ptstore_latent_attention_t* a, void* stream) {
    const char* const call = "ptstore_latent_attention";
    if (!a) return refuse_as(call, "null argument");
    LatentPlan p;
    if (const char* bad = plane_of(&a->cache, &p.kv)) return refuse_as(call, bad);
    if (const char* bad = batch_of(a->n_tokens, a->R, a->max_blocks, a->cache.block_tokens, a->heads))
        return refuse_as(call, bad);
    if (!(a->scale > 0.f) || !std::isfinite(a->scale * 1.4426950408889634f))
        return refuse_as(call, "scale must be positive and finite");
    if (a->n_tokens == 0) return PTSTORE_OK;
    if (!a->offsets || !a->context || !a->block_table) return refuse_as(call, "null argument");
    if (!rows_ok(a->q_latent, a->q_latent_token_stride, a->q_latent_head_stride) ||
        !rows_ok(a->q_rope, a->q_rope_token_stride, a->q_rope_head_stride) ||
        !rows_ok(a->out, a->out_token_stride, a->out_head_stride))
        return refuse_as(call, "rows of the queries or of out null or not 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(a->lse) & 3) return refuse_as(call, "lse not 4-byte aligned");
    // no order is promised between a row's output and the reads of other rows' queries
    if (a->out == a->q_latent || a->out == a->q_rope) return refuse_as(call, "out must be neither of the queries");
    if (p.kv.blocks < 1) return refuse_as(call, "the cache has no blocks");
    int cus = 0;
    if (const int rc = compute_units(call, &cus)) return rc;
    if (a->workspace_bytes < latent_workspace(p.kv.latent, cus) || !a->workspace || !aligned16(a->workspace))
        return refuse_as(call, "workspace too small or not 16-byte aligned (ptstore_latent_attention_workspace)");
    p.ql = Rows{a->q_latent, a->q_latent_token_stride, a->q_latent_head_stride};
    p.qr = Rows{a->q_rope, a->q_rope_token_stride, a->q_rope_head_stride};
    p.out = Rows{a->out, a->out_token_stride, a->out_head_stride};
    p.lse = a->lse;
    p.offsets = a->offsets;
    p.context = a->context;
    p.table = a->block_table;
    p.n_tokens = a->n_tokens;
    p.R = a->R;
    p.max_blocks = a->max_blocks;
    p.group = a->heads;
    p.few_rows = INT32_MAX;
    p.scale2 = a->scale * 1.4426950408889634f;
    p.parts = static_cast<float*>(a->workspace);
    p.shares = cus;
    const hipError_t e = launch_latent(p, (hipStream_t)stream);
    return e == hipSuccess ? PTSTORE_OK : set_last_error(PTSTORE_ERR_HIP, "ptstore_latent_attention: launch");
}

int ptstore_latent_expanded_workspace(int32_t heads, int64_t n_keys, int64_t* bytes) {
    // (of sizes that the call refuses there is no size, and the product could overflow)
    if (!bytes || heads < 1 || n_keys < 0 || n_keys > kMostKeys || (n_keys / 128 + 1) * heads > kMaxUnits)
        return refuse("ptstore_latent_expanded_workspace: heads or n_keys out of range, or a null argument");
    *bytes = expanded_workspace(heads, n_keys);
    return PTSTORE_OK;
}

int ptstore_latent_attention_expanded(const ptstore_latent_expanded_t* a, void* stream) {
    const char* const call = "ptstore_latent_attention_expanded";
    if (!a) return refuse_as(call, "null argument");
    ExpandedPlan p;
    if (const char* bad = plane_of(&a->cache, &p.kv)) return refuse_as(call, bad);
    if (const char* bad = batch_of(a->n_tokens, a->R, a->max_blocks, a->cache.block_tokens, a->heads))
        return refuse_as(call, bad);
    if (a->n_keys < 0 || a->n_keys > kMostKeys) return refuse_as(call, "n_keys out of range");
    if ((a->n_tokens / 128 + a->R + 1) * a->heads > kMaxUnits || (a->n_keys / 128 + 1) * a->heads > kMaxUnits)
        return refuse_as(call, "too many tiles for one call");
    if (!(a->scale > 0.f) || !std::isfinite(a->scale * 1.4426950408889634f))
        return refuse_as(call, "scale must be positive and finite");
    if (a->n_tokens == 0) return PTSTORE_OK;
    if (!a->offsets || !a->context || !a->block_table || !a->key_offsets) return refuse_as(call, "null argument");
    if (!rows_ok(a->q_nope, a->q_nope_token_stride, a->q_nope_head_stride) ||
        !rows_ok(a->q_rope, a->q_rope_token_stride, a->q_rope_head_stride) ||
        !rows_ok(a->out, a->out_token_stride, a->out_head_stride))
        return refuse_as(call, "rows of the queries or of out null or not 16-byte aligned");
    if (!rows_ok(a->w_k, a->w_k_row_stride, a->w_k_head_stride) ||
        !rows_ok(a->w_v, a->w_v_row_stride, a->w_v_head_stride))
        return refuse_as(call, "rows of w_k or w_v null or not 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(a->lse) & 3) return refuse_as(call, "lse not 4-byte aligned");
    // no order is promised between a row's output and the reads of other rows' queries
    if (a->out == a->q_nope || a->out == a->q_rope) return refuse_as(call, "out must be neither of the queries");
    if (p.kv.blocks < 1) return refuse_as(call, "the cache has no blocks");
    if (a->workspace_bytes < expanded_workspace(a->heads, a->n_keys) ||
        (a->n_keys > 0 && (!a->workspace || !aligned16(a->workspace))))
        return refuse_as(call, "workspace too small or not 16-byte aligned (ptstore_latent_expanded_workspace)");
    int cus = 0;
    if (const int rc = compute_units(call, &cus)) return rc;
    p.qn = Rows{a->q_nope, a->q_nope_token_stride, a->q_nope_head_stride};
    p.qr = Rows{a->q_rope, a->q_rope_token_stride, a->q_rope_head_stride};
    p.out = Rows{a->out, a->out_token_stride, a->out_head_stride};
    p.wk = Rows{a->w_k, a->w_k_row_stride, a->w_k_head_stride};
    p.wv = Rows{a->w_v, a->w_v_row_stride, a->w_v_head_stride};
    p.lse = a->lse;
    p.offsets = a->offsets;
    p.context = a->context;
    p.table = a->block_table;
    p.key_offsets = a->key_offsets;
    p.n_tokens = a->n_tokens;
    p.n_keys = a->n_keys;
    p.R = a->R;
    p.max_blocks = a->max_blocks;
    p.heads = a->heads;
    p.group = 1;
    p.few_rows = 0;
    p.scale2 = a->scale * 1.4426950408889634f;
    place_expanded(&p, a->workspace);
    const hipError_t e = launch_expanded(p, cus, (hipStream_t)stream);
    return e == hipSuccess ? PTSTORE_OK : set_last_error(PTSTORE_ERR_HIP, "ptstore_latent_attention_expanded: launch");
}

}  // extern "C"
#pragma GCC visibility pop
