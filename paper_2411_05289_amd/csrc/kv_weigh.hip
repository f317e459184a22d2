// The weight that every slot was given: softmax weights summed over rows, from the rows' sums that the attention left.
//
// A wave has 16 * kTiles slots of a sequence and goes through all cache heads and their rows, 16 at a time: scores are formed
// transposed, S^T = K Q^T, a lane has those of one row, and adds its weights up for each slot; the lanes that have the same slots
// meet once, in the end.  No sum is shared between waves: each has one order, whatever else runs.
#include "four_bits.h"
#include "tree_attention.h"

#include <cfloat>

namespace mdsd {

struct WeighParams {
    Cache cache;
    Scales scales;
    Trees trees;
    Heads q;
    int depth, group;
    Divisor by_group, by_tiles;
    float scale;  // times log2(e)
    const float* lse;
    const int32_t* outcome;  // NULL: all nodes
    const int32_t* accept_depth;
    const float* weights;  // NULL: zeros
    float* out;
    int64_t ld_weights, ld_out;
    int slots, tiles;  // of a row
    int32_t* flags;
};

// How many nodes the accepted path has, and which, by all threads of a workgroup (barriers inside).  path[]: the nodes, but
// of a complete tree of one branch, where node i is the i-th.
__device__ inline int find_path(const WeighParams& P, int b, int count, int* path, int* found)
{
    const Trees& R = P.trees;
    const int steps = min(P.accept_depth[b], P.depth - 1);
    const int32_t* const outcome = P.outcome + (int64_t)b * R.N;
    if (R.complete && R.k == 1) {
        // it ends behind the first outcome that is not zero
        const int most = max(0, min(steps, count - 1));
        if (threadIdx.x == 0) *found = most;
        __syncthreads();
        for (int i = threadIdx.x; i < most; i += kAttentionThreads)
            if (outcome[i] != 0) atomicMin(found, i);
        __syncthreads();
        return *found + 1;
    }
    if (threadIdx.x == 0) {
        int i = 0;
        for (int node = 0; node >= 0; ++i) {
            path[i] = node;
            node = i < steps ? next_of_path(R, node, count, outcome[node]) : -1;
        }
        *found = i;
    }
    __syncthreads();
    return *found;
}

// kDim: the head's elements, filled up to 64, 128 or 256
template <class T, int kDim, int kTiles, bool kFour>
__global__ __launch_bounds__(kAttentionThreads) void kv_weigh_kernel(WeighParams P)
{
    constexpr int kRowBytes = kDim * sizeof(T), kKeyChunks = kRowBytes / 64, kOfWave = 16 * kTiles;
    constexpr int kKeyUnit = kDim / 8 < 16 ? 8 : 16, kKeyUnits = kDim / 8 / kKeyUnit;
    extern __shared__ int nodes_of[];  // parents, or the path
    __shared__ int found;
    const Cache& C = P.cache;
    const Trees& R = P.trees;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, col = lane & 15;
    const int b = P.by_tiles((int)blockIdx.x), tile = (int)blockIdx.x - b * P.tiles;
    const int capacity = C.table_pages * C.page_size;
    const int count = R.count(b), given_length = C.lengths[b], length = min(given_length, capacity);
    const int from = tile * 4 * kOfWave, first = from + wave * kOfWave;  // the workgroup's slots, the wave's
    if (given_length < 0 && P.flags && tile == 0 && threadIdx.x == 0) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);

    const float* const weights = P.weights ? P.weights + b * P.ld_weights : nullptr;
    float* const out = P.out + b * P.ld_out;
    int nodes = length < 0 ? 0 : count;
    // (at most count nodes: the workgroups behind them have nothing to add)
    if (nodes == 0 || (int64_t)length + nodes <= from) {
        for (int s = from + threadIdx.x; s < min(from + 4 * kOfWave, P.slots); s += kAttentionThreads)
            if (out != weights) out[s] = weights ? weights[s] : 0.f;
        return;
    }
    const bool chain = R.complete && R.k == 1;
    if (P.outcome)
        nodes = find_path(P, b, count, nodes_of, &found);
    else if (!R.complete)
        parents_from_table(R, nodes_of);
    const int* const path = P.outcome && !chain ? nodes_of : nullptr;  // NULL: the i-th row's node is node i
    const int end = (int)min((int64_t)length + nodes, (int64_t)P.slots);

    // a lane looks up one slot's place; -1: it has none, or lies behind the last
    int64_t place = -1;
    {
        const int s = first + (lane & (kOfWave - 1));
        if (s < end) {
            const int i = s - length;
            place = place_of(C, C.table + b * C.ld_table, i >= 0 ? (int64_t)given_length + (path ? path[i] : i) : s);
        }
    }
    const uint64_t absent = __ballot(place < 0) & low_bits(kOfWave);
    if (P.flags && lane == 0 && (absent & low_bits(end - first))) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
    f32x4 sum[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int rows = nodes * P.group, dim_bytes = C.dim * (int)sizeof(T);
    const bool masked = first + kOfWave > length || absent != 0;
    // rows that see none of these slots come first in a chain
    const int first_row = (path || chain) && first > length ? (first - length) * P.group / 16 * 16 : 0;
    for (int kv_head = 0; kv_head < (first < end ? C.heads : 0); ++kv_head) {
        u32x4 k[kTiles][kKeyChunks];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int lo = __shfl((int)(uint32_t)place, t * 16 + col), hi = __shfl((int)(place >> 32), t * 16 + col);
            const int64_t at = kv_head * C.ld_head + (hi < 0 ? (int64_t)0 : (int64_t)hi << 32 | (uint32_t)lo);
            if constexpr (kFour) {
                constexpr int kOfUnit = kKeyUnit * 2 * sizeof(T) / 16;
                Codes<kKeyUnit> codes[kKeyUnits];
#pragma unroll
                for (int i = 0; i < kKeyUnits; ++i)
                    codes[i].load(C.k + at, P.scales.k + (at >> 4), min(quarter * (kDim / 8) + i * kKeyUnit, C.dim / 2 - kKeyUnit));
#pragma unroll
                for (int i = 0; i < kKeyChunks; ++i) k[t][i] = codes[i / kOfUnit].template chunk<T>(i % kOfUnit);
            } else {
#pragma unroll
                for (int i = 0; i < kKeyChunks; ++i) {
                    const int c = quarter * (kRowBytes / 4) + i * 16;
                    k[t][i] = *(const u32x4*)(C.k + at + min(c, dim_bytes - 16));
                    if (c >= dim_bytes) k[t][i] = u32x4{0, 0, 0, 0};
                }
            }
        }
        for (int row0 = first_row; row0 < rows; row0 += 16) {
            const int row = min(row0 + col, rows - 1), i = P.by_group(row), head = kv_head * P.group + row - i * P.group;
            const int node = path ? path[i] : i;
            const char* const q_row = P.q.p + b * P.q.ld_tree + node * P.q.ld_node + head * P.q.ld_head;
            u32x4 q[kKeyChunks];
#pragma unroll
            for (int j = 0; j < kKeyChunks; ++j) {
                const int c = quarter * (kRowBytes / 4) + j * 16;
                q[j] = u32x4{0, 0, 0, 0};
                if (c < dim_bytes) q[j] = *(const u32x4*)(q_row + c);
            }
            const float lse = P.lse[((int64_t)b * R.N + node) * P.q.heads + head];
            f32x4 s[kTiles];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < kKeyChunks; ++j) {
                    if constexpr (sizeof(T) == 4) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[t][j][e]), __uint_as_float(q[j][e]), s[t], 0, 0, 0);
                    } else {
                        s[t] = Element<T>::mfma(k[t][j], q[j], s[t]);
                    }
                }
            }
            if (masked) {
                // a path's nodes see each other as a chain's do
                int ancestor = node;
                const uint64_t seen = ~absent & (low_bits(length - first) |
                                                 (path ? low_bits(length - first + i + 1) : nodes_seen<kOfWave>(R, nodes_of, length - first, node, ancestor)));
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!(seen >> (t * 16 + quarter * 4 + e) & 1)) s[t][e] = -INFINITY;
            }
            // (a row that saw nothing adds nothing, nor does one that is not there)
            if (row0 + col < rows && lse != -INFINITY) {
                float shift = lse * 1.44269504088896f;
                if (shift == -INFINITY) shift = -FLT_MAX;  // (what is not seen stays below it)
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[t][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], P.scale, -shift));
            }
        }
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = sum[t][e];
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) x += __shfl_xor(x, d);
            const int s = first + t * 16 + quarter * 4 + e;
            if (col == 0 && s < P.slots) out[s] = (weights ? weights[s] : 0.f) + x;
        }
}

template <class T, int kDim, bool kFour>
static int weigh(WeighParams& P, hipStream_t st)
{
    constexpr int kTiles = kDim == 256 ? 2 : 4;
    const int64_t tiles = ((int64_t)P.slots + 64 * kTiles - 1) / (64 * kTiles), groups = P.trees.B * tiles;
    if (groups > kMostGroups) return MDSD_E_SHAPE;
    P.tiles = (int)tiles;
    P.by_tiles = Divisor::of(P.tiles);
    // parents of a table's nodes, or a path, which a complete tree of several branches has few of
    const size_t lds = P.trees.complete ? 64 * sizeof(int) : P.trees.N * sizeof(int);
    (void)hipGetLastError();
    hipLaunchKernelGGL((kv_weigh_kernel<T, kDim, kTiles, kFour>), dim3((unsigned)groups), dim3(kAttentionThreads), lds, st, P);
    return hipGetLastError() == hipSuccess ? MDSD_OK : MDSD_E_LAUNCH;
}
template <class T>
static int weigh(WeighParams& P, hipStream_t st)
{
    const int dim = P.cache.dim;
    if (P.scales.k) return dim <= 64 ? weigh<T, 64, true>(P, st) : dim <= 128 ? weigh<T, 128, true>(P, st) : weigh<T, 256, true>(P, st);
    return dim <= 64 ? weigh<T, 64, false>(P, st) : dim <= 128 ? weigh<T, 128, false>(P, st) : weigh<T, 256, false>(P, st);
}

}  // namespace mdsd

extern "C" int mdsd_kv_weigh(const mdsd_kv_cache* cache, const mdsd_kv_scales* scales, int32_t layer, const mdsd_tree* tree,
                             const mdsd_heads* q, const float* lse, float scale, const int32_t* outcome, const int32_t* accept_depth,
                             const float* weights, int64_t ld_weights, float* out, int64_t ld_out, int32_t slots, int32_t* flags,
                             void* stream)
{
    using namespace mdsd;
    WeighParams P = {};
    int dtype;
    int rc = check_cache(cache, scales, tree, &P.cache, &P.scales, &dtype, &P.trees);
    if (rc == kEmptyTrees) return MDSD_OK;
    if (rc != MDSD_OK) return rc;
    if ((rc = check_heads(q, P.cache, dtype, &P.q)) != MDSD_OK) return rc;
    if (!lse || !out || (outcome == nullptr) != (accept_depth == nullptr)) return MDSD_E_NULL;
    if (layer < 0 || layer >= cache->layers || q->heads % cache->heads || slots < 1 || slots > kMostSlots) return MDSD_E_SHAPE;
    if ((weights && ld_weights < slots) || ld_out < slots || ld_weights >> 46 || ld_out >> 46) return MDSD_E_SHAPE;
    const double scale_of_two = (double)scale * 1.4426950408889634;
    if (!(scale > 0.f) || !(scale_of_two <= FLT_MAX)) return MDSD_E_TEMP;
    if (((uintptr_t)lse | (uintptr_t)outcome | (uintptr_t)accept_depth | (uintptr_t)weights | (uintptr_t)out | (uintptr_t)flags) & 3)
        return MDSD_E_ALIGN;
    if (weights && rows_overlap(weights, ld_weights, out, ld_out, tree->B, slots)) return MDSD_E_ALIGN;
    if ((int64_t)tree->N * (q->heads / cache->heads) > INT32_MAX - 16) return MDSD_E_SHAPE;
    P.depth = tree->depth;
    P.group = q->heads / cache->heads;
    P.by_group = Divisor::of(P.group);
    P.scale = (float)scale_of_two;
    P.lse = lse;
    P.outcome = outcome;
    P.accept_depth = accept_depth;
    P.weights = weights;
    P.out = out;
    P.ld_weights = ld_weights;
    P.ld_out = ld_out;
    P.slots = slots;
    P.flags = flags;
    choose_layer(layer, &P.cache, &P.scales);
    hipStream_t st = (hipStream_t)stream;
    switch (dtype) {
    case MDSD_FP32: return weigh<float>(P, st);
    case MDSD_BF16: return weigh<__bf16>(P, st);
    default: return weigh<_Float16>(P, st);
    }
}
