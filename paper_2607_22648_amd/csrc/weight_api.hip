// The C calls on the weights of cached tokens (include/ptstore.h): checks on the host, launch rules, no allocation
// and no state.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "checks.hpp"
#include "ptstore.h"
#include "weights.hpp"

using namespace ptsd;

namespace {

constexpr int64_t kMaxWeighHeads = 1ll << 22;  // a workgroup a head at least, and a few for the shares' rounding
// Workgroups that move, of 256 threads: 2^31 work-items. A unit (layer, request, head) has three of them at least, and one
// of 1,024 threads that chooses: fewer than 2^32 / 1.5.
constexpr int64_t kMaxWorkgroups = 1ll << 23;

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

// What both weighing calls check and fill.
template <class Args>
const char* weigh_plan(const Args& a, int32_t q_heads, int32_t block_tokens, WeighPlan* p) {
    if (const char* bad = batch_of(a.n_tokens, a.R, a.max_blocks, block_tokens, q_heads)) return bad;
    if (p->kv.heads >= kMaxWeighHeads) return "too many heads for one call (2^22 or more)";
    if (!(a.scale > 0.f) || !std::isfinite(a.scale * 1.4426950408889634f)) return "scale must be positive and finite";
    if (a.n_tokens == 0) return nullptr;
    if (!a.offsets || !a.context || !a.block_table || !a.lse || !a.weights) return "null argument";
    if (!aligned4(a.lse) || !aligned4(a.weights)) return "lse or weights not 4-byte aligned";
    if (p->kv.blocks < 1) return "the cache has no blocks";
    p->lse = a.lse;
    p->offsets = a.offsets;
    p->context = a.context;
    p->weighed = a.weighed;
    p->table = a.block_table;
    p->n_tokens = a.n_tokens;
    p->R = a.R;
    p->max_blocks = a.max_blocks;
    p->q_heads = q_heads;
    p->group = q_heads / p->kv.heads;
    p->rows_div = page_div(p->group);
    p->scale2 = a.scale * 1.4426950408889634f;
    p->weights = a.weights;
    p->parts = static_cast<float*>(a.workspace);
    return nullptr;
}

template <class Args>
int weigh(const char* call, const Args& a, WeighPlan* p, void* stream) {
    int cus = 0;
    if (const int rc = compute_units(call, &cus)) return rc;
    if (a.workspace_bytes < weigh_workspace(p->kv.heads, cus) || !a.workspace || !aligned16(a.workspace))
        return refuse_as(call, "workspace too small or not 16-byte aligned (ptstore_weigh_workspace)");
    p->cus = cus;
    return launch_weigh(*p, (hipStream_t)stream) == hipSuccess ? PTSTORE_OK : set_last_error(PTSTORE_ERR_HIP, call);
}

// What both evicting calls check and fill; the plan's planes are there.
int evict(const char* call, const ptstore_evict_t* a, KeepPlan* p, int64_t plane_bytes, void* stream) {
    if (!a) return refuse_as(call, "null argument");
    if (a->layers < 0 || a->R < 0 || a->max_blocks < 1 || (int64_t)a->R * a->max_blocks > kMaxEntries ||
        a->max_keep < 0 || a->recent < 0)
        return refuse_as(call, "layers, R, max_blocks, max_keep or recent out of range");
    if ((int64_t)a->max_blocks * p->div.page > kMaxKeys) return refuse_as(call, "max_blocks * block_tokens exceeds 2^30");
    if (a->layers == 0 || a->R == 0) return PTSTORE_OK;
    if (a->layer_bytes % 16 || (a->layers > 1 && a->layer_bytes < plane_bytes))
        return refuse_as(call, "layer_bytes must be a multiple of 16 and hold a layer's planes");
    p->layer = a->layer_bytes;
    p->slab_rows = page_div(p->heads * (int)p->div.page);
    p->layers = a->layers;
    p->R = a->R;
    p->max_blocks = a->max_blocks;
    if ((double)a->layers * a->R * p->heads > (double)kMaxWorkgroups || keep_workgroups(*p) > kMaxWorkgroups)
        return refuse_as(call, "too many layers, requests and heads for one call");
    if (!a->weights || !a->context || !a->keep || !a->context_out || !a->block_table || !a->to_table)
        return refuse_as(call, "null argument");
    if (!aligned4(a->weights)) return refuse_as(call, "weights not 4-byte aligned");
    if (a->context_out == a->context || a->context_out == a->keep)
        return refuse_as(call, "context_out must be neither context nor keep");
    if (p->blocks < 1) return refuse_as(call, "the cache has no blocks");
    int64_t need = 0;
    if (ptstore_evict_workspace(a->layers, a->R, p->heads, a->max_keep, &need) != PTSTORE_OK)
        return refuse_as(call, "max_keep out of range");
    if (a->workspace_bytes < need || (need > 0 && (!a->workspace || !aligned16(a->workspace))))
        return refuse_as(call, "workspace too small or not 16-byte aligned (ptstore_evict_workspace)");
    p->weights = a->weights;
    p->context = a->context;
    p->keep = a->keep;
    p->context_out = a->context_out;
    p->from = a->block_table;
    p->to = a->to_table;
    p->max_keep = a->max_keep;
    p->recent = a->recent;
    p->source = static_cast<int32_t*>(a->workspace);
    int cus = 0;
    if (const int rc = compute_units(call, &cus)) return rc;
    return launch_keep(*p, cus, (hipStream_t)stream) == hipSuccess ? PTSTORE_OK : set_last_error(PTSTORE_ERR_HIP, call);
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int ptstore_weigh_workspace(int32_t kv_heads, int64_t* bytes) {
    const char* const call = "ptstore_weigh_workspace";
    if (!bytes || kv_heads < 1 || kv_heads >= kMaxWeighHeads) return refuse_as(call, "kv_heads out of range, or a null argument");
    int cus = 0;
    if (const int rc = compute_units(call, &cus)) return rc;
    *bytes = weigh_workspace(kv_heads, cus);
    return PTSTORE_OK;
}

int ptstore_kv_weigh(const ptstore_weigh_t* a, void* stream) {
    const char* const call = "ptstore_kv_weigh";
    if (!a) return refuse_as(call, "null argument");
    WeighPlan p{};
    if (const char* bad = planes_of(&a->kv, &p.kv)) return refuse_as(call, bad);
    if (a->q_heads < 1 || a->q_heads % a->kv.kv_heads) return refuse_as(call, "q_heads must be a multiple of the cache's heads");
    if (const char* bad = weigh_plan(*a, a->q_heads, a->kv.block_tokens, &p)) return refuse_as(call, bad);
    if (a->n_tokens == 0) return PTSTORE_OK;
    if (!rows_ok(a->q, a->q_token_stride, a->q_head_stride)) return refuse_as(call, "rows of q null or not 16-byte aligned");
    p.q = Rows{a->q, a->q_token_stride, a->q_head_stride};
    return weigh(call, *a, &p, stream);
}

int ptstore_latent_weigh(const ptstore_latent_weigh_t* a, void* stream) {
    const char* const call = "ptstore_latent_weigh";
    if (!a) return refuse_as(call, "null argument");
    WeighPlan p{};
    if (const char* bad = plane_of(&a->cache, &p.latent)) return refuse_as(call, bad);
    p.is_latent = true;
    p.kv.heads = 1;
    p.kv.blocks = p.latent.blocks;
    p.kv.div = p.latent.div;
    if (const char* bad = weigh_plan(*a, a->heads, a->cache.block_tokens, &p)) return refuse_as(call, bad);
    if (a->n_tokens == 0) return PTSTORE_OK;
    if (!rows_ok(a->q_latent, a->q_latent_token_stride, a->q_latent_head_stride) ||
        !rows_ok(a->q_rope, a->q_rope_token_stride, a->q_rope_head_stride))
        return refuse_as(call, "rows of the queries null or not 16-byte aligned");
    p.q = Rows{a->q_latent, a->q_latent_token_stride, a->q_latent_head_stride};
    p.qr = Rows{a->q_rope, a->q_rope_token_stride, a->q_rope_head_stride};
    return weigh(call, *a, &p, stream);
}

int ptstore_evict_workspace(int32_t layers, int32_t R, int32_t kv_heads, int32_t max_keep, int64_t* bytes) {
    if (!bytes || layers < 0 || R < 0 || kv_heads < 1 || max_keep < 0 ||
        (double)layers * R * kv_heads > (double)kMaxWorkgroups)
        return refuse("ptstore_evict_workspace: a size is out of range, or a null argument");
    *bytes = ((int64_t)layers * R * kv_heads * max_keep * 4 + 15) / 16 * 16;
    return PTSTORE_OK;
}

int ptstore_kv_evict(const ptstore_kv_t* kv, const ptstore_evict_t* a, void* stream) {
    const char* const call = "ptstore_kv_evict";
    Planes pl;
    if (const char* bad = planes_of(kv, &pl)) return refuse_as(call, bad);
    const bool four = pl.kind == PTSTORE_KV_MXFP4;
    KeepPlan p{};
    p.k = pl.k;
    p.v = pl.v;
    p.blocks = pl.blocks;
    p.heads = pl.heads;
    p.div = pl.div;
    p.slab = pl.slab;
    p.row = four ? pl.dim / 2 : pl.dim * 2;
    p.power = four ? pl.dim / kGroup : 0;
    p.powers = pl.exponents;
    return evict(call, a, &p, 2 * pl.blocks * (int64_t)pl.slab, stream);
}

int ptstore_latent_evict(const ptstore_latent_t* cache, const ptstore_evict_t* a, void* stream) {
    const char* const call = "ptstore_latent_evict";
    LatentPlane pl;
    if (const char* bad = plane_of(cache, &pl)) return refuse_as(call, bad);
    KeepPlan p{};
    p.k = pl.rows;
    p.blocks = pl.blocks;
    p.heads = 1;
    p.div = pl.div;
    p.row = (int32_t)pl.line * 16;
    p.slab = (int64_t)pl.div.page * p.row;
    return evict(call, a, &p, pl.blocks * p.slab, stream);
}

}  // extern "C"
#pragma GCC visibility pop
