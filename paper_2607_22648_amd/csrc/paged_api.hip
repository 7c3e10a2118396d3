// The C calls of the paged cache's operators (include/ptstore.h): checks on the
// host, launch rules, no allocation and no state.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "checks.hpp"
#include "paged.hpp"
#include "ptstore.h"

namespace ptsd {

static int64_t slab_bytes(int32_t kind, int32_t heads, int32_t dim, int32_t page) {
    if (heads < 1 || (dim != 64 && dim != 128) || page < 1 || page > 64) return -1;
    const int64_t rows = (int64_t)heads * page;
    int64_t n;
    if (kind == PTSTORE_KV_BF16 || kind == PTSTORE_KV_FP16)
        n = rows * dim * 2;
    else if (kind == PTSTORE_KV_MXFP4)
        n = (rows * (dim / 2 + dim / kGroup) + 15) / 16 * 16;
    else
        return -1;
    return n <= 1ll << 30 ? n : -1;
}

// The planes of `kv`, or a message.
const char* planes_of(const ptstore_kv_t* kv, Planes* out) {
    if (!kv) return "null cache";
    const int64_t slab = slab_bytes(kv->kind, kv->kv_heads, kv->head_dim, kv->block_tokens);
    if (slab < 0) return "the cache's kind, heads, head_dim (64, 128) or block_tokens (1..64) is not supported";
    if (kv->cache_blocks < 0 || kv->cache_blocks > kMaxCacheBlocks) return "cache_blocks out of range (0..2^30)";
    if (kv->cache_blocks * slab > kMaxPlane) return "a plane of the cache exceeds 64 GiB";
    if (kv->cache_blocks > 0 && (!kv->k || !kv->v || !aligned16(kv->k) || !aligned16(kv->v)))
        return "the cache's planes must be 16-byte aligned";
    out->k = static_cast<uint8_t*>(kv->k);
    out->v = static_cast<uint8_t*>(kv->v);
    out->blocks = kv->cache_blocks;
    out->heads = kv->kv_heads;
    out->dim = kv->head_dim;
    out->div = page_div(kv->block_tokens);
    out->slab = (uint32_t)slab;
    out->exponents = (uint32_t)(kv->kv_heads * kv->block_tokens * (kv->head_dim / 2));
    out->kind = kv->kind;
    return nullptr;
}

}  // namespace ptsd

using namespace ptsd;

namespace {

constexpr int64_t kMaxUnits = kMaxItems / 256 - 8192;  // (tile, KV head) pairs of prompt.hip, and room for
                                                       // parts of the last ones
constexpr int64_t kMaxHeads = kMaxItems / 512;         // decode.hip: a workgroup a head at least, 512 threads

// Whether a call's rows go 128 to a tile, or 16. The host knows the average
// request alone. Behind 4,000 keys, 8 KV heads of 4 query heads (us, joins included):
//
//   tokens x requests   4 x 32  16 x 32  32 x 32   64 x 2  128 x 2  256 x 2
//   16 rows                 91      252      525       55       86      167
//   128 rows               149      150      156       38       43       68
bool many_rows(const AttendPlan& p) { return p.n_tokens * p.group > (int64_t)32 * p.R; }

// Whether a batch goes to both kernels, requests of few rows to the one for 16 and the
// others to the one for 128. A workgroup of the latter goes through all keys of a tile,
// 1.3 us for 64, however few its rows are; in the former a long request reads its keys
// once for each 16 rows: 256 single tokens and 512 tokens of one request, behind
// 4,000, take 745 us by both and 905 by the former. The launches that may find nothing to
// do cost 5 to 9 us (64 drafts of 4 tokens: 170 us, 162), so it takes room for 8,192 keys
// and, in a batch of few rows a request, kManyRows beyond a token each: at 508 of them
// both ways take the same time (256 single tokens and 128 of one request, 720 us). The room
// is the table's, not the requests': in a wide table every batch of several prompts pays for
// the launches (4 prompts of 256 tokens take 19.1 us beside 14.2 in a tight one).
constexpr int64_t kManyRows = 512;
bool mixed(const AttendPlan& p, bool prompts) {
    return p.R > 1 && (int64_t)p.max_blocks * p.kv.div.page >= 8192 &&
           (prompts || (p.n_tokens - p.R) * p.group >= kManyRows);
}

int64_t workspace_of(const Planes& kv, int cus) {
    const int64_t a = decode_workspace(kv, decode_shares(kv, cus)), b = prompt_workspace(kv, cus);
    return a > b ? a : b;
}

// Checks the sizes and fills what the workspace and the launch follow from.
const char* sized(const ptstore_kv_t* kv, int32_t q_heads, int64_t n_tokens, int32_t R, int32_t max_blocks,
                  AttendPlan* p) {
    if (const char* bad = planes_of(kv, &p->kv)) return bad;
    if (q_heads < 1 || q_heads % kv->kv_heads) return "q_heads must be a multiple of the cache's heads";
    if (R < 0 || max_blocks < 1 || (int64_t)R * max_blocks > kMaxEntries || n_tokens < 0 ||
        (R == 0 && n_tokens > 0))
        return "R, max_blocks or n_tokens out of range";
    if ((int64_t)max_blocks * kv->block_tokens > kMaxKeys) return "max_blocks * block_tokens exceeds 2^30";
    if (kv->kv_heads >= kMaxHeads) return "too many heads for one call (2^23 or more)";
    // rows are numbered in 32 bits, up to the end of a last tile
    constexpr int64_t most = (1ll << 31) - kPromptRows;
    if (n_tokens > most || n_tokens * q_heads > most) return "n_tokens * q_heads exceeds 2^31 - 128";
    p->n_tokens = n_tokens;
    p->R = R;
    p->max_blocks = max_blocks;
    p->q_heads = q_heads;
    p->group = q_heads / kv->kv_heads;
    const bool prompts = many_rows(*p);
    if ((prompts || mixed(*p, prompts)) &&
        tile_bound(n_tokens, p->group, R, kPromptRows) * kv->kv_heads > kMaxUnits)
        return "too many tiles for one call";
    return nullptr;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int ptstore_kv_slab_bytes(int32_t kind, int32_t kv_heads, int32_t head_dim, int32_t block_tokens,
                          int64_t* bytes) {
    const int64_t n = slab_bytes(kind, kv_heads, head_dim, block_tokens);
    if (n < 0 || !bytes) return refuse("ptstore_kv_slab_bytes: kind, heads, head_dim (64, 128) or block_tokens "
                                       "(1..64) not supported, or a slab over 1 GiB");
    *bytes = n;
    return PTSTORE_OK;
}

int ptstore_block_tables(const int64_t* offsets, int64_t n_tokens, const int32_t* context, const int32_t* held,
                         int32_t R, int32_t max_blocks, int32_t block_tokens, const int32_t* free_blocks,
                         int64_t n_free, const int64_t* first, int32_t* block_table, int64_t* slots,
                         int32_t* positions, int32_t* held_out, int64_t* next, void* stream) {
    if (R < 0 || max_blocks < 1 || (int64_t)R * max_blocks > kMaxEntries || block_tokens < 1 ||
        block_tokens > 64 || (int64_t)max_blocks * block_tokens > kMaxKeys || n_tokens < 0 ||
        n_tokens >= (1ll << 40) || n_free < 0 || (R == 0 && n_tokens > 0))
        return refuse("ptstore_block_tables: a size is out of range");
    if (!next || (R > 0 && (!offsets || !context || !block_table || !held_out)) || (n_tokens > 0 && !slots) ||
        (n_free > 0 && !free_blocks))
        return refuse("ptstore_block_tables: null argument");
    // every workgroup reads them while one writes
    if (held_out == held && held) return refuse("ptstore_block_tables: held_out must not be held");
    if (next == first) return refuse("ptstore_block_tables: next must not be first");
    TablesPlan p{offsets, n_tokens, context,     held,  R,         max_blocks, page_div(block_tokens), free_blocks,
                 n_free,  first,    block_table, slots, positions, held_out,   next};
    const hipError_t e = launch_tables(p, (hipStream_t)stream);
    return e == hipSuccess ? PTSTORE_OK : set_last_error(PTSTORE_ERR_HIP, "ptstore_block_tables: launch");
}

static int move_rows(const char* call, const ptstore_kv_t* kv, const void* k, int64_t k_token, int64_t k_head,
                     const void* v, int64_t v_token, int64_t v_head, const int64_t* slots, int64_t n,
                     bool read, void* stream) {
    Planes pl;
    if (const char* bad = planes_of(kv, &pl)) return refuse_as(call, bad);
    // a work-item moves 8 elements; the last workgroup may be partly filled
    if (n < 0 || n > (kMaxItems - 256) / (pl.dim / 8) / pl.heads)
        return refuse_as(call, "n_tokens * kv_heads * head_dim exceeds 2^35 - 2^11");
    if (n == 0) return PTSTORE_OK;
    if (!slots || !rows_ok(k, k_token, k_head) || !rows_ok(v, v_token, v_head))
        return refuse_as(call, "null argument, or rows of k or v not 16-byte aligned");
    const Rows kr{k, k_token, k_head}, vr{v, v_token, v_head};
    const hipError_t e = read ? launch_read(pl, kr, vr, slots, n, (hipStream_t)stream)
                              : launch_append(pl, kr, vr, slots, n, (hipStream_t)stream);
    return e == hipSuccess ? PTSTORE_OK : set_last_error(PTSTORE_ERR_HIP, call);
}

int ptstore_kv_append(const ptstore_kv_t* kv, const void* k, int64_t k_token_stride, int64_t k_head_stride,
                      const void* v, int64_t v_token_stride, int64_t v_head_stride, const int64_t* slots,
                      int64_t n_tokens, void* stream) {
    return move_rows("ptstore_kv_append", kv, k, k_token_stride, k_head_stride, v, v_token_stride,
                     v_head_stride, slots, n_tokens, false, stream);
}

int ptstore_kv_read(const ptstore_kv_t* kv, void* k, int64_t k_token_stride, int64_t k_head_stride, void* v,
                    int64_t v_token_stride, int64_t v_head_stride, const int64_t* slots, int64_t n_tokens,
                    void* stream) {
    return move_rows("ptstore_kv_read", kv, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride,
                     slots, n_tokens, true, stream);
}

int ptstore_attention_workspace(const ptstore_kv_t* kv, int64_t* bytes) {
    Planes pl;
    if (!bytes) return refuse("ptstore_attention_workspace: null argument");
    if (const char* bad = planes_of(kv, &pl)) return refuse_as("ptstore_attention_workspace", bad);
    int cus = 0;
    if (const int rc = compute_units("ptstore_attention", &cus)) return rc;
    *bytes = workspace_of(pl, cus);
    return PTSTORE_OK;
}

int ptstore_attention(const ptstore_attention_t* a, void* stream) {
    if (!a) return refuse("ptstore_attention: null argument");
    AttendPlan p;
    if (const char* bad = sized(&a->kv, a->q_heads, a->n_tokens, a->R, a->max_blocks, &p))
        return refuse_as("ptstore_attention", bad);
    if (!(a->scale > 0.f) || !std::isfinite(a->scale * 1.4426950408889634f))
        return refuse("ptstore_attention: scale must be positive and finite");
    if (a->n_tokens == 0) return PTSTORE_OK;
    if (!a->offsets || !a->context || !a->block_table) return refuse("ptstore_attention: null argument");
    if (!rows_ok(a->q, a->q_token_stride, a->q_head_stride) ||
        !rows_ok(a->out, a->out_token_stride, a->out_head_stride))
        return refuse("ptstore_attention: rows of q or out null or not 16-byte aligned");
    // no order is promised between a row's output and the reads of other rows' queries
    if (a->out == a->q) return refuse("ptstore_attention: out must not be q");
    if (p.kv.blocks < 1) return refuse("ptstore_attention: the cache has no blocks");
    int cus = 0;
    if (const int rc = compute_units("ptstore_attention", &cus)) return rc;
    if (a->workspace_bytes < workspace_of(p.kv, cus) || !a->workspace || !aligned16(a->workspace))
        return refuse("ptstore_attention: workspace too small or not 16-byte aligned "
                      "(ptstore_attention_workspace)");
    p.q = Rows{a->q, a->q_token_stride, a->q_head_stride};
    p.out = Rows{a->out, a->out_token_stride, a->out_head_stride};
    p.lse = a->lse;
    p.offsets = a->offsets;
    p.context = a->context;
    p.table = a->block_table;
    p.scale2 = a->scale * 1.4426950408889634f;
    p.parts = static_cast<float*>(a->workspace);
    p.shares = decode_shares(p.kv, cus);
    const bool prompts = many_rows(p), both = mixed(p, prompts);
    hipError_t e = hipSuccess;
    if (prompts || both) {
        p.few_rows = both ? kFewRows : 0;
        split_prompt(&p, cus);
        e = launch_prompt(p, (hipStream_t)stream);
    }
    if (e == hipSuccess && (!prompts || both)) {
        p.few_rows = both ? kFewRows : INT32_MAX;
        e = launch_decode(p, (hipStream_t)stream);
    }
    return e == hipSuccess ? PTSTORE_OK : set_last_error(PTSTORE_ERR_HIP, "ptstore_attention: launch");
}

}  // extern "C"
#pragma GCC visibility pop
