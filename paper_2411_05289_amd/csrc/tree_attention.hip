// Attention of tree nodes: checks and launches.
#include "tree_attention.h"

namespace mdsd {

template <class T, int kDim>
static int launch(const AttentionParams& P, hipStream_t st)
{
    const int64_t groups = (int64_t)P.trees.B * P.row_tiles * P.cache.heads;
    if (groups > INT32_MAX) return MDSD_E_SHAPE;
    const size_t lds = AttentionTile<T, kDim>::kLds + (P.trees.complete ? 0 : P.trees.N * sizeof(int));
    (void)hipGetLastError();
    if (hipFuncSetAttribute((const void*)tree_attention_kernel<T, kDim>, hipFuncAttributeMaxDynamicSharedMemorySize,
                            (int)lds) != hipSuccess)
        return MDSD_E_LAUNCH;
    hipLaunchKernelGGL((tree_attention_kernel<T, kDim>), dim3((unsigned)groups), dim3(kAttentionThreads), lds, st, P);
    return hipGetLastError() == hipSuccess ? MDSD_OK : MDSD_E_LAUNCH;
}

template <class T>
static int launch_by_dim(const AttentionParams& P, hipStream_t st)
{
    if (P.cache.dim <= 64) return launch<T, 64>(P, st);
    if (P.cache.dim <= 128) return launch<T, 128>(P, st);
    return launch<T, 256>(P, st);
}

}  // namespace mdsd

extern "C" {

size_t mdsd_tree_attention_workspace_bytes(const mdsd_kv_cache* cache, const mdsd_tree* tree, int32_t q_heads,
                                           int32_t shared, int32_t longest)
{
    return 0;
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
    P.group = q->heads / cache->heads;
    const int64_t rows = (int64_t)tree->N * P.group;
    if (rows > INT32_MAX - kRowsOfTile) return MDSD_E_SHAPE;
    P.row_tiles = (int)((rows + kRowsOfTile - 1) / kRowsOfTile);
    P.by_group = Divisor::of(P.group);
    P.scale = (float)((double)scale * 1.4426950408889634);
    P.shared_pages = shared_pages;
    P.shared = shared;
    P.flags = flags;
    P.cache.k += layer * P.cache.ld_layer;
    P.cache.v += layer * P.cache.ld_layer;
    hipStream_t st = (hipStream_t)stream;
    switch (cache->dtype) {
    case MDSD_FP32: return launch_by_dim<float>(P, st);
    case MDSD_BF16: return launch_by_dim<__bf16>(P, st);
    default: return launch_by_dim<_Float16>(P, st);
    }
}

}  // extern "C"
