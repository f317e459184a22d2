// The weight that every slot was given: softmax weights summed over rows, from the rows' sums that the attention left.
//
// A workgroup has some slots of a sequence and goes through all cache heads and their rows, 16 at a time: scores are formed
// transposed, S^T = K Q^T, a lane has those of one row, and adds its weights up for each slot; the lanes and waves that have the
// same slots meet once, in the end, in one order whatever else runs.
//
// What bounds it is reading the keys, once: the accepted paths of 64 trees behind 512 to 4096 slots, 306 MB of bf16 keys, 70.1 us, 4.4 TB/s;
// 64 tokens behind 1024 to 16384 slots in 4 bits, 304 MB, 74 us, 4.1 TB/s, beside 50 us of vector instructions; one
// token behind 16384 slots 6 us, of which an empty launch is 3; 32 fp32 trees of 15 nodes behind 512 to 4096 slots, 9 GFLOP, in 4 bits 113 us, in 32 202.
// Prompts of 512 tokens behind 2048 to 4096 slots, 56 GFLOP, 129 us: queries from the L2.
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
    int lds_shifts, lds_nodes;  // of few rows: where these stand in LDS
    int32_t* flags;
};

// Sum over the 16 lanes of a row of lanes, by data-parallel moves
__device__ inline float sum_of_row(float x)
{
    auto turned = [](float y, auto control) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), decltype(control)::value, 0xf, 0xf, false));
    };
    x += turned(x, std::integral_constant<int, 0x121>());
    x += turned(x, std::integral_constant<int, 0x122>());
    x += turned(x, std::integral_constant<int, 0x124>());
    x += turned(x, std::integral_constant<int, 0x128>());
    return x;
}

// Leaves out of a row's scores the slots that it does not see; `seen`: a bit for each.  A row whose sum is no number
// gives none to what it sees, and nothing to the rest: its scores then say so, and what all of them are lowered by must not.
template <int kTiles>
__device__ inline void leave_out(f32x4 (&s)[kTiles], uint64_t seen, int quarter, float lse)
{
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!(seen >> (t * 16 + quarter * 4 + e) & 1)) s[t][e] = -INFINITY;
    // (hardly ever; prompts of 512 tokens 129 us, and 136 by an addition for each score)
    if (lse != lse) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (seen >> (t * 16 + quarter * 4 + e) & 1) s[t][e] = lse;
    }
}

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
        for (int i = threadIdx.x; i < most; i += blockDim.x)
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

// kDim: the head's elements, filled up to 64, 128 or 256.  The waves of a workgroup go through the same 16 * kTiles slots, each
// with its share of the cache heads.  What bounds many rows is reading the queries, once for every workgroup, from the L2.
template <class Given, int kDim, int kTiles, int kWaves, bool kFour>
__global__ __launch_bounds__(64 * kWaves) void kv_weigh_kernel(WeighParams P)
{
    using T = Worked<Given, kFour>;
    constexpr int kParts = kPartsOf<Given, kFour>;
    constexpr int kRowBytes = kDim * sizeof(T), kKeyChunks = kRowBytes / 64, kSlots = 16 * kTiles;
    constexpr int kKeyUnit = kDim / 8 < 16 ? 8 : 16, kKeyUnits = kDim / 8 / kKeyUnit;
    extern __shared__ int nodes_of[];  // parents, or the path
    __shared__ int found;
    __shared__ __attribute__((aligned(16))) float sums[kWaves][kSlots];
    const Cache& C = P.cache;
    const Trees& R = P.trees;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, col = lane & 15;
    const int b = P.by_tiles((int)blockIdx.x), tile = (int)blockIdx.x - b * P.tiles;
    const int capacity = C.table_pages * C.page_size;
    const int count = R.count(b), given_length = C.lengths[b], length = min(given_length, capacity);
    const int first = tile * kSlots;
    if (given_length < 0 && P.flags && tile == 0 && threadIdx.x == 0) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);

    const float* const weights = P.weights ? P.weights + b * P.ld_weights : nullptr;
    float* const out = P.out + b * P.ld_out;
    int nodes = length < 0 ? 0 : count;
    // (at most count nodes: the workgroups behind them have nothing to add)
    if (nodes == 0 || (int64_t)length + nodes <= first) {
        const int s = first + threadIdx.x;
        if ((int)threadIdx.x < kSlots && s < P.slots && out != weights) out[s] = weights ? weights[s] : 0.f;
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
        const int s = first + (lane & (kSlots - 1));
        if (s < end) {
            const int i = s - length;
            place = place_of(C, C.table + b * C.ld_table, i >= 0 ? (int64_t)given_length + (path ? path[i] : i) : s);
        }
    }
    const uint64_t absent = __ballot(place < 0) & low_bits(kSlots);
    if (P.flags && lane == 0 && (absent & low_bits(end - first))) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
    int64_t key_at[kTiles];  // of the lane's keys
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const int lo = __shfl((int)(uint32_t)place, t * 16 + col), hi = __shfl((int)(place >> 32), t * 16 + col);
        key_at[t] = hi < 0 ? (int64_t)0 : (int64_t)hi << 32 | (uint32_t)lo;
    }
    f32x4 sum[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int rows = nodes * P.group, dim_bytes = C.dim * (int)sizeof(T);
    const bool masked = first + kSlots > length || absent != 0;
    // rows that see none of these slots come first in a chain
    const int first_row = (path || chain) && first > length ? (first - length) * P.group / 16 * 16 : 0;
    const int head_end = first < end && first_row < rows ? C.heads : 0;

    // Keys of the next head and queries of the next rows are asked for while these are worked on
    u32x4 keys[kTiles][kKeyChunks];
    Codes<kKeyUnit, false> codes[kTiles][kKeyUnits];  // (in 4 bits, in place of the above)
    auto load_keys = [&](int kv_head) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int64_t at = key_at[t] + kv_head * C.ld_head;
            if constexpr (kFour) {
#pragma unroll
                for (int i = 0; i < kKeyUnits; ++i)
                    codes[t][i].load(C.k + at, P.scales.k + (at >> 4), min(quarter * (kDim / 8) + i * kKeyUnit, C.dim / 2 - kKeyUnit));
            } else {
#pragma unroll
                for (int i = 0; i < kKeyChunks; ++i) {
                    const int c = quarter * 16 + i * 64;  // (a key's four lanes side by side)
                    keys[t][i] = *(const u32x4*)(C.k + at + min(c, dim_bytes - 16));
                    if (c >= dim_bytes) keys[t][i] = u32x4{0, 0, 0, 0};
                }
            }
        }
    };
    struct Row {
        int i, node;  // of the rows' nodes, and in the tree
        float lse;
        u32x4 q[kKeyChunks][kParts];
    } next;
    auto load_row = [&](int kv_head, int row0) {
        const int row = min(row0 + col, rows - 1);
        next.i = P.by_group(row);
        next.node = path ? path[next.i] : next.i;
        const int head = kv_head * P.group + row - next.i * P.group;
        const char* const q_row = P.q.p + b * P.q.ld_tree + next.node * P.q.ld_node + head * P.q.ld_head;
#pragma unroll
        for (int j = 0; j < kKeyChunks; ++j) {
            const int c = kFour ? quarter * (kRowBytes / 4) + j * 16 : quarter * 16 + j * 64;
#pragma unroll
            for (int p = 0; p < kParts; ++p) next.q[j][p] = u32x4{0, 0, 0, 0};
            if (c < dim_bytes) {
                if constexpr (kParts == 3)
                    in_parts((const float*)(q_row + 2 * c), next.q[j]);
                else
                    next.q[j][0] = *(const u32x4*)(q_row + c);
            }
        }
        next.lse = P.lse[((int64_t)b * R.N + next.node) * P.q.heads + head];
    };
    int kv_head = wave;
    if (kv_head < head_end) {
        load_keys(kv_head);
        load_row(kv_head, first_row);
    }
    for (; kv_head < head_end; kv_head += kWaves) {
        u32x4 k[kTiles][kKeyChunks];
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int i = 0; i < kKeyChunks; ++i) {
                if constexpr (kFour) {
                    constexpr int kOfUnit = kKeyUnit * 2 * sizeof(T) / 16;
                    k[t][i] = codes[t][i / kOfUnit].template chunk<T>(i % kOfUnit);
                } else {
                    k[t][i] = keys[t][i];
                }
            }
        if (kv_head + kWaves < head_end) load_keys(kv_head + kWaves);
        for (int row0 = first_row; row0 < rows; row0 += 16) {
            const Row row = next;
            if (row0 + 16 < rows)
                load_row(kv_head, row0 + 16);
            else if (kv_head + kWaves < head_end)
                load_row(kv_head + kWaves, first_row);
            f32x4 s[kTiles];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < kKeyChunks; ++j) {
                    if constexpr (sizeof(T) == 4) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[t][j][e]), __uint_as_float(row.q[j][0][e]), s[t], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int p = 0; p < kParts; ++p) s[t] = Element<T>::mfma(k[t][j], row.q[j][p], s[t]);
                    }
                }
            }
            if (masked) {
                // a path's nodes see each other as a chain's do
                int ancestor = row.node;
                const uint64_t seen = ~absent & (low_bits(length - first) |
                                                 (path ? low_bits(length - first + row.i + 1)
                                                       : nodes_seen<kSlots>(R, nodes_of, length - first, row.node, ancestor)));
                leave_out(s, seen, quarter, row.lse);
            }
            // (a row that saw nothing adds nothing, nor does one that is not there)
            if (row0 + col < rows && row.lse != -INFINITY) {
                float shift = row.lse * 1.44269504088896f;
                if (shift == -INFINITY) shift = -FLT_MAX;  // (what is not seen stays below it)
                if (masked && shift != shift) shift = 0.f;  // (see leave_out)
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[t][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], P.scale, -shift));
            }
        }
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[t][e] = sum_of_row(sum[t][e]);
        if (col == 0) *(f32x4*)&sums[wave][t * 16 + quarter * 4] = sum[t];
    }
    __syncthreads();
    const int s = first + threadIdx.x;
    if ((int)threadIdx.x < kSlots && s < P.slots) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x += sums[w][threadIdx.x];
        out[s] = (weights ? weights[s] : 0.f) + x;
    }
}

constexpr int64_t kMostWorkgroups = kMostGroups / 2;  // of four waves as of eight, so that it does not hang on the kernel

template <class T, int kDim, int kTiles, int kWaves, bool kFour>
static int launch_weigh(WeighParams& P, hipStream_t st)
{
    const int64_t tiles = ((int64_t)P.slots + 16 * kTiles - 1) / (16 * kTiles), groups = P.trees.B * tiles;
    if (groups > kMostWorkgroups) return MDSD_E_SHAPE;
    P.tiles = (int)tiles;
    P.by_tiles = Divisor::of(P.tiles);
    // parents of a table's nodes, or a path, which a complete tree of several branches has few of
    const size_t lds = P.trees.complete ? 64 * sizeof(int) : P.trees.N * sizeof(int);
    (void)hipGetLastError();
    hipLaunchKernelGGL((kv_weigh_kernel<T, kDim, kTiles, kWaves, kFour>), dim3((unsigned)groups), dim3(64 * kWaves), lds, st, P);
    return hipGetLastError() == hipSuccess ? MDSD_OK : MDSD_E_LAUNCH;
}
// For few rows: all of them, of every cache head, stand in LDS, so that memory has nothing to give but keys, and a wave goes
// through its kOfWave slots, 16 * kTiles at a time, with the keys of kAhead heads on their way.
template <class Given, int kDim, int kTiles, int kAhead, int kOfWave, bool kFour>
__global__ __launch_bounds__(kAttentionThreads) void kv_weigh_few_kernel(WeighParams P)
{
    using T = Worked<Given, kFour>;
    constexpr int kParts = kPartsOf<Given, kFour>;
    constexpr int kRowBytes = kDim * sizeof(T), kKeyChunks = kRowBytes / 64, kChunks = kRowBytes / 16, kSlots = 16 * kTiles;
    constexpr int kKeyUnit = kDim / 8 < 16 ? 8 : 16, kKeyUnits = kDim / 8 / kKeyUnit;
    extern __shared__ __attribute__((aligned(16))) char lds[];  // the rows' chunks, [part][row][chunk]; their shifts; a path or parents
    __shared__ int found;
    __shared__ __attribute__((aligned(16))) float sums[4][kOfWave];
    const Cache& C = P.cache;
    const Trees& R = P.trees;
    float* const shifts = (float*)(lds + P.lds_shifts);
    int* const nodes_of = (int*)(lds + P.lds_nodes);
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
        const int s = from + threadIdx.x;
        if (threadIdx.x < 4 * kOfWave && s < P.slots && out != weights) out[s] = weights ? weights[s] : 0.f;
        return;
    }
    const bool chain = R.complete && R.k == 1;
    if (P.outcome)
        nodes = find_path(P, b, count, nodes_of, &found);
    else if (!R.complete)
        parents_from_table(R, nodes_of);
    const int* const path = P.outcome && !chain ? nodes_of : nullptr;  // NULL: the i-th row's node is node i
    const int end = (int)min((int64_t)length + nodes, (int64_t)P.slots);
    const int rows = nodes * P.group, all_rows = rows * C.heads, dim_bytes = C.dim * (int)sizeof(T);

    // a lane looks up one slot's place; -1: it has none, or lies behind the last
    int64_t place = -1;
    const int own = first + lane;
    if (lane < kOfWave && own < end) {
        const int i = own - length;
        place = place_of(C, C.table + b * C.ld_table, i >= 0 ? (int64_t)given_length + (path ? path[i] : i) : own);
    }
    const uint64_t absent = __ballot(place < 0);
    if (P.flags && lane == 0 && (absent & low_bits(min(end - first, kOfWave)))) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);

    // the wave's slots and heads in one line
    u32x4 keys[kAhead][kTiles][kKeyChunks];
    Codes<kKeyUnit, false> codes[kAhead][kTiles][kKeyUnits];  // (in 4 bits, in place of the above)
    const int steps = first < end ? (min(end - first, kOfWave) + kSlots - 1) / kSlots * C.heads : 0;
    int next_slots = 0, next_head = 0;  // of the next keys that are asked for
    auto load_keys = [&](int at) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int of = next_slots + t * 16 + col;
            const int lo = __shfl((int)(uint32_t)place, of), hi = __shfl((int)(place >> 32), of);
            const int64_t from = next_head * C.ld_head + (hi < 0 ? (int64_t)0 : (int64_t)hi << 32 | (uint32_t)lo);
            if constexpr (kFour) {
#pragma unroll
                for (int i = 0; i < kKeyUnits; ++i)
                    codes[at][t][i].load(C.k + from, P.scales.k + (from >> 4), min(quarter * (kDim / 8) + i * kKeyUnit, C.dim / 2 - kKeyUnit));
            } else {
#pragma unroll
                for (int i = 0; i < kKeyChunks; ++i) {
                    const int c = quarter * 16 + i * 64;  // (a key's four lanes side by side)
                    keys[at][t][i] = *(const u32x4*)(C.k + from + min(c, dim_bytes - 16));
                }
            }
        }
        if (++next_head == C.heads) {
            next_head = 0;
            next_slots = (next_slots + kSlots) & (kOfWave - 1);  // (behind the last: some keys that nobody looks at)
        }
    };
    auto first_keys = [&] {
        if (steps) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) load_keys(j);
        }
    };
    // (paths of 64 sequences in 16 bits 72.1 us, 70.5; 16 tokens behind 16384 slots in 4 bits 38.8, 40.3, where they come after the rows)
    if constexpr (!kFour) first_keys();
    // row r of cache head h is row h * rows + r here; its chunks are turned by its number against bank conflicts
    for (int i = threadIdx.x; i < all_rows * kChunks; i += kAttentionThreads) {
        const int row = i / kChunks, c = i % kChunks, h = row / rows, r = row - h * rows, n = P.by_group(r);
        const int node = path ? path[n] : n, head = h * P.group + r - n * P.group;
        const char* const q_row = P.q.p + b * P.q.ld_tree + node * P.q.ld_node + head * P.q.ld_head;
        u32x4 x[kParts];
#pragma unroll
        for (int p = 0; p < kParts; ++p) x[p] = u32x4{0, 0, 0, 0};
        if (c * 16 < dim_bytes) {
            if constexpr (kParts == 3)
                in_parts((const float*)(q_row + c * 32), x);
            else
                x[0] = *(const u32x4*)(q_row + c * 16);
        }
#pragma unroll
        for (int p = 0; p < kParts; ++p) *(u32x4*)(lds + ((p * all_rows + row) * kChunks + (c ^ (row & (kChunks - 1)))) * 16) = x[p];
        if (c == 0) {
            // what a row's scores are lowered by; minus infinity: a row that saw nothing adds nothing
            const float lse = P.lse[((int64_t)b * R.N + node) * P.q.heads + head], shift = lse * 1.44269504088896f;
            shifts[row] = lse != -INFINITY && shift == -INFINITY ? -FLT_MAX : shift;
        }
    }
    if constexpr (kFour) first_keys();
    __syncthreads();
    const float before = weights && lane < kOfWave && own < P.slots ? weights[own] : 0.f;

    int at_slots = 0, kv_head = 0;
    f32x4 sum[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int step0 = 0; step0 < steps; step0 += kAhead) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (step0 + j >= steps) break;
            u32x4 k[kTiles][kKeyChunks];
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int i = 0; i < kKeyChunks; ++i) {
                    if constexpr (kFour) {
                        constexpr int kOfUnit = kKeyUnit * 2 * sizeof(T) / 16;
                        k[t][i] = codes[j][t][i / kOfUnit].template chunk<T>(i % kOfUnit);
                    } else {
                        k[t][i] = keys[j][t][i];
                        if (quarter * 16 + i * 64 >= dim_bytes) k[t][i] = u32x4{0, 0, 0, 0};
                    }
                }
            load_keys(j);
            const int here = first + at_slots;
            const uint64_t absent_here = absent >> at_slots & low_bits(kSlots);
            const bool masked = here + kSlots > length || absent_here != 0;
            // rows that see none of these slots come first in a chain
            for (int row0 = (path || chain) && here > length ? (here - length) * P.group / 16 * 16 : 0; row0 < rows; row0 += 16) {
                const int r = min(row0 + col, rows - 1), row = kv_head * rows + r;
                float shift = shifts[row];
                f32x4 s[kTiles];
#pragma unroll
                for (int t = 0; t < kTiles; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < kKeyChunks; ++i) {
                    const int c = kFour ? quarter * kKeyChunks + i : quarter + i * 4;
#pragma unroll
                    for (int p = 0; p < kParts; ++p) {
                        const u32x4 q = *(const u32x4*)(lds + ((p * all_rows + row) * kChunks + (c ^ (row & (kChunks - 1)))) * 16);
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) {
                            if constexpr (sizeof(T) == 4) {
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[t][i][e]), __uint_as_float(q[e]), s[t], 0, 0, 0);
                            } else {
                                s[t] = Element<T>::mfma(k[t][i], q, s[t]);
                            }
                        }
                    }
                }
                if (masked) {
                    // a path's nodes see each other as a chain's do
                    const int n = P.by_group(r), node = path ? path[n] : n;
                    int ancestor = node;
                    const uint64_t seen = ~absent_here & (low_bits(length - here) |
                                                          (path ? low_bits(length - here + n + 1)
                                                                : nodes_seen<kSlots>(R, nodes_of, length - here, node, ancestor)));
                    leave_out(s, seen, quarter, shift);
                    shift = shift != shift ? 0.f : shift;
                }
                if (row0 + col < rows && shift != -INFINITY) {
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[t][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], P.scale, -shift));
                }
            }
            if (++kv_head < C.heads) continue;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[t][e] = sum_of_row(sum[t][e]);
                if (col == 0) *(f32x4*)&sums[wave][at_slots + t * 16 + quarter * 4] = sum[t];
                sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            kv_head = 0;
            at_slots += kSlots;
        }
    }
    // (its own wave's)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (lane < kOfWave && own < P.slots) out[own] = before + (lane < at_slots ? sums[wave][lane] : 0.f);
}

template <class T, int kDim, bool kFour>
static int weigh(WeighParams& P, hipStream_t st)
{
    const Trees& R = P.trees;
    const bool path = P.outcome && !(R.complete && R.k == 1);
    const int64_t rows = (int64_t)(path && R.complete ? min(P.depth, R.N) : R.N) * P.group, all = rows * P.cache.heads;
    const size_t bytes = sizeof(Worked<T, kFour>) * kDim * kPartsOf<T, kFour>;
    const size_t nodes = R.complete ? 64 * sizeof(int) : R.N * sizeof(int);
    // The rows in LDS, where three workgroups' fit and there are slots enough to fill the chip 256 a workgroup (us, without and with: bf16
    // keys in 4 bits, 32 heads over 8 of 128: a token of 1 sequence behind 16384 slots 5.8, 14.2, of 4 15.4, 16.5, of 8 27.2, 20.8,
    // of 16 60.3, 39.6; the paths of 16 sequences of up to 4096 15.9, 26.6, of 64 in 16 bits 101, 70).  What is known here is the width of the
    // weights, not the lengths: a token behind 16384 slots takes 6.0 us with weights of up to 98304 slots, and 13.8 with 131072.
    if (all * bytes <= 48 * 1024 && (int64_t)R.B * P.slots > 98304) {
        P.lds_shifts = (int)(all * bytes);
        P.lds_nodes = P.lds_shifts + (int)all * 4;
        constexpr int kTiles = kFour ? 2 : 1, kAhead = 2;
        const size_t lds = P.lds_nodes + nodes;  // (at most 384 rows, and nodes: below 52 KB, so that no limit is to be asked for)
        const auto launch = [&](auto of_wave) -> int {
            constexpr int kOfWave = decltype(of_wave)::value;
            const int64_t tiles = ((int64_t)P.slots + 4 * kOfWave - 1) / (4 * kOfWave), groups = R.B * tiles;
            if (groups > kMostWorkgroups) return MDSD_E_SHAPE;
            P.tiles = (int)tiles;
            P.by_tiles = Divisor::of(P.tiles);
            const auto kernel = kv_weigh_few_kernel<T, kDim, kTiles, kAhead, kOfWave, kFour>;
            (void)hipGetLastError();
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(kAttentionThreads), lds, st, P);
            return hipGetLastError() == hipSuccess ? MDSD_OK : MDSD_E_LAUNCH;
        };
        // Half as many slots where three workgroups a compute unit would not be full, and reading takes all the time (a token of 8 sequences
        // behind 16384 slots of bf16 67 us, 53; in 4 bits 20.4, 21.6; of 64 tokens of up to 16384 in 4 bits 73.5, 74.3)
        if constexpr (!kFour)
            if (R.B * (((int64_t)P.slots + 255) / 256) < 768) return launch(std::integral_constant<int, 32>());
        return launch(std::integral_constant<int, 64>());
    }
    // 64 slots a wave where many rows pay for them (prompts of 512 tokens, us by 16, 32, 64: 477, 291, 224; a token 8.5, 6.7, 8.2, in 16
    // bits 11.9, 13.9, 17.2), and eight waves for as many heads (226, 126; fp32 has no registers for them)
    if (rows > 64) {
        constexpr int kMany = kDim == 256 ? 2 : 4;
        if constexpr (sizeof(T) == 2)
            if (P.cache.heads >= 8) return launch_weigh<T, kDim, kMany, 8, kFour>(P, st);
        return launch_weigh<T, kDim, kMany, 4, kFour>(P, st);
    }
    return launch_weigh<T, kDim, kFour ? 2 : 1, 4, kFour>(P, st);
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
