// Attention of tree nodes: checks, and how a call is cut into launches.
#include "tree_attention_plan.h"

namespace mdsd {

constexpr int kComputeUnits = 256;

static int padded_dim(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

static bool plan_attention(const mdsd_kv_cache* c, const mdsd_tree* t, int q_heads, int shared, int longest, bool workspace,
                           AttentionPlan* plan)
{
    AttentionPlan& p = *plan;
    p = AttentionPlan{};
    const int G = q_heads / c->heads, size = c->dtype == MDSD_FP32 ? 4 : 2, row_bytes = padded_dim(c->dim) * size;
    p.rows = (int64_t)t->N * G;
    if (p.rows > INT32_MAX - kJointRows) return false;
    p.tile_rows = p.rows <= 16 ? 16 : p.rows <= 32 ? 32 : p.rows <= 64 && row_bytes <= 512 ? 64 : 128;
    p.row_tiles = (int)((p.rows + p.tile_rows - 1) / p.tile_rows);
    p.units = (int64_t)t->B * p.row_tiles * c->heads;
    if (p.units > INT32_MAX) return false;
    if (!workspace) return true;
    const int64_t capacity = (int64_t)c->table_pages * c->page_size;
    const int64_t most = (longest ? (longest < capacity ? longest : capacity) : capacity) + t->N;
    const bool joint = shared >= 256 && t->B > 1 && p.row_tiles == 1 && (int64_t)t->B * p.rows <= INT32_MAX - kJointRows;
    const int per_unit = row_bytes <= 256 ? 2 : 1;
    const int slots = kComputeUnits * per_unit;
    // (a cache head's tiles are counted in 32 bits)
    if ((!joint && (p.units >= 4 * slots || most <= 256)) || p.units / c->heads * (capacity / 32 + 1) > INT32_MAX) return true;
    p.groups = slots;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t from = at;
        at += (bytes + 255) / 256 * 256;
        return from;
    };
    auto parts = [&](int64_t units, int groups, int rows, size_t* ends, size_t* stats, size_t* sums) {
        *ends = take(units * 8);
        *stats = take((size_t)(units + groups) * rows * 8);
        *sums = take((size_t)(units + groups) * rows * c->dim * 4);
    };
    parts(p.units, p.groups, p.tile_rows, &p.ends, &p.stats, &p.sums);
    if (joint) {
        p.joint_tiles = (int)((t->B * p.rows + kJointRows - 1) / kJointRows);
        p.joint_groups = kComputeUnits * per_unit;
        parts((int64_t)p.joint_tiles * c->heads, p.joint_groups, kJointRows, &p.joint_ends, &p.joint_stats, &p.joint_sums);
    }
    p.bytes = at;
    return true;
}

}  // namespace mdsd

extern "C" {

size_t mdsd_tree_attention_workspace_bytes(const mdsd_kv_cache* cache, const mdsd_tree* tree, int32_t q_heads,
                                           int32_t shared, int32_t longest)
{
    using namespace mdsd;
    Cache C;
    Trees T;
    AttentionPlan plan;
    if (check_cache(cache, tree, &C, &T) != MDSD_OK || q_heads < 1 || q_heads % cache->heads || shared < 0 || longest < 0)
        return 0;
    return plan_attention(cache, tree, q_heads, shared, longest, true, &plan) ? plan.bytes : 0;
}

int mdsd_tree_attention(const mdsd_kv_cache* cache, int32_t layer, const mdsd_tree* tree, const mdsd_heads* q,
                        const mdsd_heads* out, float scale, const int32_t* shared_pages, int32_t shared,
                        int32_t longest, int32_t* flags, void* ws, size_t ws_bytes, void* stream)
{
    using namespace mdsd;
    AttentionParams P = {};
    int rc = check_cache(cache, tree, &P.cache, &P.trees);
    if (rc == kEmptyTrees) return MDSD_OK;
    if (rc != MDSD_OK) return rc;
    if ((rc = check_heads(q, P.cache, cache->dtype, &P.q)) != MDSD_OK) return rc;
    if ((rc = check_heads(out, P.cache, cache->dtype, &P.out)) != MDSD_OK) return rc;
    if (layer < 0 || layer >= cache->layers) return MDSD_E_SHAPE;
    if (q->heads != out->heads || q->heads % cache->heads) return MDSD_E_SHAPE;
    if (shared < 0 || longest < 0 || shared > (int64_t)cache->table_pages * cache->page_size) return MDSD_E_SHAPE;
    if (shared && !shared_pages) return MDSD_E_NULL;
    if (!(scale > 0.f) || scale > 3.0e38f) return MDSD_E_TEMP;
    if ((uintptr_t)flags & 3 || (uintptr_t)shared_pages & 3 || (uintptr_t)ws & 15) return MDSD_E_ALIGN;
    AttentionPlan plan;
    if (!plan_attention(cache, tree, q->heads, shared, longest, ws != nullptr, &plan)) return MDSD_E_SHAPE;
    if (ws_bytes < plan.bytes) return MDSD_E_WORKSPACE;
    P.group = q->heads / cache->heads;
    P.by_group = Divisor::of(P.group);
    P.by_heads = Divisor::of(cache->heads);
    P.by_rows = Divisor::of((int)plan.rows);
    P.scale = (float)((double)scale * 1.4426950408889634);
    P.slack = fminf(8.f / P.scale, 1e30f);
    P.shared_pages = shared_pages;
    P.shared = shared;
    P.flags = flags;
    P.cache.k += layer * P.cache.ld_layer;
    P.cache.v += layer * P.cache.ld_layer;
    hipStream_t st = (hipStream_t)stream;
    switch (cache->dtype) {
    case MDSD_FP32: return attend_fp32(cache->dim, P, plan, (char*)ws, st);
    case MDSD_BF16: return attend_bf16(cache->dim, P, plan, (char*)ws, st);
    default: return attend_fp16(cache->dim, P, plan, (char*)ws, st);
    }
}

}  // extern "C"
