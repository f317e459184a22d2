// The accepted path of every tree: its keys and values move to where the sequence goes on.
//
// One workgroup per sequence and layer.  The path's i-th node n >= i moves from slot length + n to slot length + i; a
// thread moves one 16-byte chunk of every slot of the path, in the path's order, so that a slot is written only when
// what it held is no longer needed.  What bounds it is the way to the first byte: length, path, pages, keys (64 sequences of
// 31 nodes, 32 layers of 8 heads of 128: 24 MB in 9.2 us, 2.6 TB/s; of 256 sequences 3.5 TB/s; of one 4.3 us).  Following the
// path in LDS changed nothing.
#include "kv_cache.h"

namespace mdsd {

struct CommitParams {
    Cache cache;
    Scales scales;  // of a cache in 4 bits
    Trees trees;
    int depth, chunks;  // 16-byte chunks of a head
    Divisor by_chunks, by_layer;
    const int32_t* outcome;
    const int32_t* accept_depth;
    int32_t* new_lengths;  // NULL: not by this launch
    int32_t* flags;
};

constexpr int kCommitThreads = 256, kPathPart = 64, kMostAhead = 8;

// (a sequence far behind its table stays one: a sum that wrapped round would be a sequence without nodes)
__device__ inline int new_length(int length, int nodes) { return min(length, INT32_MAX - nodes) + nodes; }

// kFour: scales move too, a byte a thread (64 paths in 32 layers of 8 heads of 128 11.7 us, in bf16 12.2; of one tree 5.4, 4.2).  As a part of
// every build they took a wave of eight from each SIMD: 64 paths in 16 bits 8.5 us, 8.8.
template <bool kFour>
__global__ __launch_bounds__(kCommitThreads) void kv_commit_kernel(CommitParams P)
{
    __shared__ int path[kPathPart], path_end;  // the part's nodes; how many of them there are
    __shared__ int64_t from[kPathPart], to[kPathPart];
    const Cache& C = P.cache;
    const int b = P.by_layer((int)blockIdx.x), own_layer = (int)blockIdx.x - b * C.layers;
    const int count = P.trees.count(b), length = C.lengths[b];
    if (length < 0 || count == 0) {
        if (threadIdx.x == 0 && own_layer == 0) {
            if (P.new_lengths) P.new_lengths[b] = length;
            if (length < 0 && P.flags) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
        }
        return;
    }
    const int32_t* const outcome = P.outcome + (int64_t)b * P.trees.N;
    const int32_t* const table = C.table + b * C.ld_table;
    const int steps = min(P.accept_depth[b], P.depth - 1);
    const int64_t layer = own_layer * C.ld_layer;
    int node = 0;
    for (int done = 0; node >= 0; done += kPathPart) {
        if (threadIdx.x == 0) {
            int i = 0;
            for (; i < kPathPart && node >= 0; ++i) {
                path[i] = node;
                node = done + i < steps ? next_of_path(P.trees, node, count, outcome[node]) : -1;
            }
            path_end = i;
        }
        __syncthreads();
        const int in_part = path_end;
        if ((int)threadIdx.x < in_part) {
            const int i = done + threadIdx.x, n = path[threadIdx.x];
            int64_t source = -1, target = -1;
            if (n != i) {
                source = place_of(C, table, (int64_t)length + n);
                target = place_of(C, table, (int64_t)length + i);
                if ((source < 0 || target < 0) && P.flags) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
            }
            from[threadIdx.x] = target < 0 ? -1 : source;  // -1: nothing moves
            to[threadIdx.x] = target;
        }
        // the first thread's node goes on; the others only need to know whether there is one
        if (threadIdx.x == 0) path[0] = node;
        __syncthreads();
        node = path[0];
        for (int item = threadIdx.x; item < 2 * C.heads * P.chunks; item += kCommitThreads) {
            const int h2 = P.by_chunks(item), c = item - h2 * P.chunks;
            char* const base = (h2 & 1 ? C.v : C.k) + layer + (h2 >> 1) * C.ld_head + c * 16;
            for (int i = 0; i < in_part; i += kMostAhead) {
                u32x4 x[kMostAhead];
#pragma unroll
                for (int j = 0; j < kMostAhead; ++j)
                    if (i + j < in_part && from[i + j] >= 0) x[j] = *(const u32x4*)(base + from[i + j]);
#pragma unroll
                for (int j = 0; j < kMostAhead; ++j)
                    if (i + j < in_part && from[i + j] >= 0) *(u32x4*)(base + to[i + j]) = x[j];
            }
        }
        if constexpr (kFour) {
            // a byte for every chunk
            const int64_t first = layer >> 4;
            for (int item = threadIdx.x; item < 2 * C.heads * P.chunks; item += kCommitThreads) {
                const int h2 = P.by_chunks(item), c = item - h2 * P.chunks;
                uint8_t* const base = (h2 & 1 ? P.scales.v : P.scales.k) + first + (h2 >> 1) * (C.ld_head >> 4) + c;
                for (int i = 0; i < in_part; i += kMostAhead) {
                    uint8_t x[kMostAhead];
#pragma unroll
                    for (int j = 0; j < kMostAhead; ++j)
                        if (i + j < in_part && from[i + j] >= 0) x[j] = base[from[i + j] >> 4];
#pragma unroll
                    for (int j = 0; j < kMostAhead; ++j)
                        if (i + j < in_part && from[i + j] >= 0) base[to[i + j] >> 4] = x[j];
                }
            }
        }
        if (node < 0 && P.new_lengths && own_layer == 0 && threadIdx.x == 0) P.new_lengths[b] = new_length(length, done + in_part);
        __syncthreads();
    }
}

// The new lengths alone, in place: one thread per sequence.
__global__ void kv_commit_lengths_kernel(CommitParams P)
{
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= P.trees.B) return;
    const int count = P.trees.count(b), length = P.new_lengths[b];
    if (length < 0 || count == 0) return;
    const int steps = min(P.accept_depth[b], P.depth - 1);
    int nodes = 0;
    for (int node = 0; node >= 0; ++nodes)
        node = nodes < steps ? next_of_path(P.trees, node, count, P.outcome[(int64_t)b * P.trees.N + node]) : -1;
    P.new_lengths[b] = new_length(length, nodes);
}

static int commit(const mdsd_kv_cache* cache, const mdsd_kv_scales* scales, const mdsd_tree* tree, const int32_t* outcome,
                  const int32_t* accept_depth, int32_t* new_lengths, int32_t* flags, void* stream)
{
    CommitParams P = {};
    int dtype;
    const int rc = check_cache(cache, scales, tree, &P.cache, &P.scales, &dtype, &P.trees);
    if (rc == kEmptyTrees) return MDSD_OK;
    if (rc != MDSD_OK) return rc;
    if (!outcome || !accept_depth || !new_lengths) return MDSD_E_NULL;
    if (((uintptr_t)outcome | (uintptr_t)accept_depth | (uintptr_t)new_lengths | (uintptr_t)flags) & 3) return MDSD_E_ALIGN;
    if (new_lengths != cache->lengths && new_lengths < cache->lengths + tree->B && cache->lengths < new_lengths + tree->B) return MDSD_E_ALIGN;
    if (one_place(*cache)) return MDSD_E_SHAPE;
    const int row = scales ? cache->dim / 2 : cache->dim * (dtype == MDSD_FP32 ? 4 : 2);  // bytes of a head
    if ((int64_t)tree->B * cache->layers > kMostGroups || (int64_t)2 * cache->heads * row / 16 > INT32_MAX - kCommitThreads) return MDSD_E_SHAPE;
    P.depth = tree->depth;
    P.chunks = row / 16;
    P.by_chunks = Divisor::of(P.chunks);
    P.by_layer = Divisor::of(cache->layers);
    P.outcome = outcome;
    P.accept_depth = accept_depth;
    P.flags = flags;
    hipStream_t st = (hipStream_t)stream;
    // every workgroup of a sequence reads its length: it changes behind them
    const bool in_place = new_lengths == cache->lengths;
    P.new_lengths = in_place ? nullptr : new_lengths;
    (void)hipGetLastError();
    hipLaunchKernelGGL(scales ? kv_commit_kernel<true> : kv_commit_kernel<false>, dim3((unsigned)(cache->layers * tree->B)), dim3(kCommitThreads), 0, st, P);
    if (hipGetLastError() != hipSuccess) return MDSD_E_LAUNCH;
    if (in_place) {
        P.new_lengths = new_lengths;
        hipLaunchKernelGGL(kv_commit_lengths_kernel, dim3((unsigned)((tree->B + 255) / 256)), dim3(256), 0, st, P);
        if (hipGetLastError() != hipSuccess) return MDSD_E_LAUNCH;
    }
    return MDSD_OK;
}

}  // namespace mdsd

extern "C" {

int mdsd_kv_commit(const mdsd_kv_cache* cache, const mdsd_tree* tree, const int32_t* outcome, const int32_t* accept_depth,
                   int32_t* new_lengths, int32_t* flags, void* stream)
{
    return mdsd::commit(cache, nullptr, tree, outcome, accept_depth, new_lengths, flags, stream);
}

int mdsd_kv4_commit(const mdsd_kv_cache* cache, const mdsd_kv_scales* scales, const mdsd_tree* tree, const int32_t* outcome,
                    const int32_t* accept_depth, int32_t* new_lengths, int32_t* flags, void* stream)
{
    if (tree && tree->B != 0 && !scales) return MDSD_E_NULL;
    return mdsd::commit(cache, scales, tree, outcome, accept_depth, new_lengths, flags, stream);
}

}  // extern "C"
