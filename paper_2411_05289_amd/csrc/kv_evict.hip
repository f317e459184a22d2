// Sequences cut to the slots that matter: which those are, and their way to the front.
//
// Two launches.  `select`: a workgroup per sequence finds the weight of the last slot that is kept by its digits, the highest
// first (three counts of 11, 11 and 10 bits), and then goes through the slots once, in order, giving each that is kept its
// new place.  `move`: what is kept only moves to the front, so that a workgroup that reads some rows in a row before it
// writes them overwrites nothing that is read later; it has one or more heads of keys or values in one layer to itself.
#include "kv_cache.h"

namespace mdsd {

struct EvictParams {
    Cache cache;
    Scales scales;
    const float* weights;
    float* weights_out;  // NULL: not asked for
    int64_t ld_weights, ld_out;
    int slots, budget, first, recent;
    int32_t* new_lengths;
    int32_t* kept;
    int32_t* flags;
    // of a move's workgroup: heads, 16-byte chunks of a head and of all of them, rows that its threads have at once
    int heads, chunks, width, rows;
    Divisor by_layer, by_part, by_width, by_chunks;
    int parts;  // of a layer: of keys and of values
};

constexpr int kSelectThreads = 1024, kDigits = 2048, kEach = 4, kMoveThreads = 256, kMoveAhead = 8;

// Whole numbers in the weights' order; NaN is the least, and the zeros are one
__device__ inline uint32_t rank_of(float x)
{
    if (x != x) return 0;
    const uint32_t bits = __float_as_uint(x + 0.f);
    return bits >> 31 ? ~bits : bits | 0x80000000u;
}

// Sum over the threads before this one, and over all; `sums`: one for each wave (barriers inside)
__device__ inline int sum_before(int x, int* sums, int* all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int up = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(up, d);
        if (lane >= d) up += y;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = up;
    __syncthreads();
    int before = 0, total = 0;
    for (int w = 0; w < kSelectThreads / 64; ++w) {
        const int of = sums[w];
        before += w < wave ? of : 0;
        total += of;
    }
    *all = total;
    return before + up - x;
}

__global__ __launch_bounds__(kSelectThreads) void kv_select_kernel(EvictParams P)
{
    __shared__ int counts[kDigits], sums[kSelectThreads / 64];
    __shared__ uint32_t chosen;
    __shared__ int chosen_left;
    const Cache& C = P.cache;
    const int b = blockIdx.x, capacity = C.table_pages * C.page_size;
    const int given = C.lengths[b], length = min(given, capacity);
    const float* const weights = P.weights + b * P.ld_weights;
    float* const out = P.weights_out ? P.weights_out + b * P.ld_out : nullptr;
    int32_t* const kept = P.kept + (int64_t)b * P.budget;
    auto weight_of = [&](int s) { return s < P.slots ? weights[s] : 0.f; };
    if (P.flags && threadIdx.x == 0 && (given < 0 || given > capacity)) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
    __syncthreads();  // (the length is read by all before it is written)
    if (threadIdx.x == 0) P.new_lengths[b] = min(length, P.budget);
    if (length <= P.budget) {
        for (int i = threadIdx.x; i < P.budget; i += kSelectThreads) kept[i] = i < length ? i : -1;
        if (out)
            for (int s = threadIdx.x; s < P.slots; s += kSelectThreads) out[s] = s < length ? weights[s] : 0.f;
        return;
    }
    const int last = length - P.recent;  // slots first .. last-1 are chosen from
    int left = P.budget - P.first - P.recent;
    uint32_t border = 0;  // ranks above it are kept, and `left` of those that are it
    if (left > 0) {
        uint32_t known = 0;
        for (int shift = 21; shift >= 0; shift = shift ? (shift == 21 ? 10 : 0) : -1) {
            const int bits = shift ? 11 : 10;
            for (int i = threadIdx.x; i < kDigits; i += kSelectThreads) counts[i] = 0;
            __syncthreads();
            for (int s = P.first + threadIdx.x; s < last; s += kSelectThreads) {
                const uint32_t r = rank_of(weight_of(s));
                if (((r ^ border) & known) == 0) atomicAdd(&counts[r >> shift & ((1 << bits) - 1)], 1);
            }
            __syncthreads();
            // digits from the highest on: thread i has 2047 - 2i and the one below it
            const int high = kDigits - 1 - 2 * (int)threadIdx.x, n0 = counts[high], n1 = counts[high - 1];
            int all;
            const int before = sum_before(n0 + n1, sums, &all);
            if (before < left && before + n0 + n1 >= left) {
                const bool upper = before + n0 >= left;
                chosen = (uint32_t)(upper ? high : high - 1);
                chosen_left = left - before - (upper ? 0 : n0);
            }
            __syncthreads();
            border |= chosen << shift;
            known |= (uint32_t)((1 << bits) - 1) << shift;
            left = chosen_left;
            __syncthreads();
        }
    }
    // the places of what is kept, kEach slots a thread at a time
    const bool none = P.budget == P.first + P.recent;
    int number = 0, equal = 0;  // kept, and at the border, so far
    for (int from = 0; from < length; from += kSelectThreads * kEach) {
        const int s0 = from + threadIdx.x * kEach;
        float w[kEach];
        bool stays[kEach], borders[kEach];
        int of_border = 0, of_kept = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int s = s0 + j;
            w[j] = s < length ? weight_of(s) : 0.f;
            const bool open = s >= P.first && s < last;
            const uint32_t r = rank_of(w[j]);
            borders[j] = open && !none && r == border;
            stays[j] = s < length && (!open || (!none && r > border));
            of_border += borders[j];
        }
        int all;
        int at = equal + sum_before(of_border, sums, &all);
        equal += all;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (borders[j]) stays[j] = at++ < left;
            of_kept += stays[j];
        }
        at = number + sum_before(of_kept, sums, &all);
        number += all;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (!stays[j]) continue;
            kept[at] = s0 + j;
            // (every thread has its weights by now, and what comes later stands behind all of these places)
            if (out && at < P.slots) out[at] = w[j];
            ++at;
        }
    }
    __syncthreads();
    if (out)
        for (int s = P.budget + threadIdx.x; s < P.slots; s += kSelectThreads) out[s] = 0.f;
}

template <bool kFour>
__global__ __launch_bounds__(kMoveThreads) void kv_move_kernel(EvictParams P)
{
    constexpr int kMostRows = kMoveThreads * kMoveAhead;
    __shared__ int64_t from[kMostRows], to[kMostRows];
    const Cache& C = P.cache;
    const int bl = P.by_part((int)blockIdx.x), part = (int)blockIdx.x - bl * P.parts, b = P.by_layer(bl), layer = bl - b * C.layers;
    const int32_t* const kept = P.kept + (int64_t)b * P.budget;
    const int32_t* const table = C.table + b * C.ld_table;
    if (kept[P.budget - 1] < P.budget) return;  // nothing moves: shorter, or as long (a slot never moves up)
    // the first that moves
    int lo = P.first, hi = P.budget - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (kept[mid] == mid)
            lo = mid + 1;
        else
            hi = mid;
    }
    const int at_row = P.by_width((int)threadIdx.x), item = threadIdx.x - at_row * P.width;
    const int of_keys = P.parts / 2, h0 = (part < of_keys ? part : part - of_keys) * P.heads, h1 = P.by_chunks(item);
    const bool mine = at_row < P.rows && h0 + h1 < C.heads;
    const int64_t column = layer * C.ld_layer + (h0 + h1) * C.ld_head + (item - h1 * P.chunks) * 16;
    char* const base = (part < of_keys ? C.k : C.v) + column;
    uint8_t* const scale = kFour ? (part < of_keys ? P.scales.k : P.scales.v) + (column >> 4) : nullptr;
    const int batch = P.rows * kMoveAhead;
    for (int i0 = lo; i0 < P.budget; i0 += batch) {
        __syncthreads();  // the places before these are read no more
        for (int i = threadIdx.x; i < batch; i += kMoveThreads) {
            int64_t source = -1, target = -1;
            if (i0 + i < P.budget) {
                source = place_of(C, table, kept[i0 + i]);
                target = place_of(C, table, i0 + i);
                if (P.flags && part == 0 && layer == 0 && (source < 0 || target < 0)) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
            }
            from[i] = target < 0 ? -1 : source;
            to[i] = target;
        }
        __syncthreads();
        u32x4 x[kMoveAhead];
        uint8_t y[kMoveAhead];
#pragma unroll
        for (int j = 0; j < kMoveAhead; ++j) {
            const int64_t source = mine ? from[at_row + j * P.rows] : -1;
            if (source >= 0) {
                x[j] = *(const u32x4*)(base + source);
                if (kFour) y[j] = scale[source >> 4];
            }
        }
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();  // all have read
#pragma unroll
        for (int j = 0; j < kMoveAhead; ++j) {
            const int64_t source = mine ? from[at_row + j * P.rows] : -1;
            if (source >= 0) {
                const int64_t target = to[at_row + j * P.rows];
                *(u32x4*)(base + target) = x[j];
                if (kFour) scale[target >> 4] = y[j];
            }
        }
    }
}

}  // namespace mdsd

extern "C" int mdsd_kv_evict(const mdsd_kv_cache* cache, const mdsd_kv_scales* scales, int32_t B, const float* weights,
                             int64_t ld_weights, int32_t slots, int32_t budget, int32_t first, int32_t recent, int32_t* new_lengths,
                             int32_t* kept, float* weights_out, int64_t ld_out, int32_t* flags, void* stream)
{
    using namespace mdsd;
    if (B == 0) return MDSD_OK;
    EvictParams P = {};
    int dtype;
    const int rc = check_pages(cache, scales, &P.cache, &P.scales, &dtype);
    if (rc != MDSD_OK) return rc;
    if (!weights || !new_lengths || !kept) return MDSD_E_NULL;
    if (B < 0 || slots < 1 || slots > kMostSlots || budget < 1 || budget > kMostSlots || first < 0 || recent < 0 ||
        (int64_t)first + recent > budget)
        return MDSD_E_SHAPE;
    if (ld_weights < slots || ld_weights >> 46 || (weights_out && (ld_out < slots || ld_out >> 46))) return MDSD_E_SHAPE;
    if (((uintptr_t)weights | (uintptr_t)new_lengths | (uintptr_t)kept | (uintptr_t)weights_out | (uintptr_t)flags) & 3) return MDSD_E_ALIGN;
    if (new_lengths != cache->lengths && new_lengths < cache->lengths + B && cache->lengths < new_lengths + B) return MDSD_E_ALIGN;
    if (weights_out && rows_overlap(weights, ld_weights, weights_out, ld_out, B, slots)) return MDSD_E_ALIGN;
    if (one_place(*cache)) return MDSD_E_SHAPE;
    P.weights = weights;
    P.weights_out = weights_out;
    P.ld_weights = ld_weights;
    P.ld_out = ld_out;
    P.slots = slots;
    P.budget = budget;
    P.first = first;
    P.recent = recent;
    P.new_lengths = new_lengths;
    P.kept = kept;
    P.flags = flags;
    const int row = scales ? cache->dim / 2 : cache->dim * (dtype == MDSD_FP32 ? 4 : 2);  // bytes of a head
    P.chunks = row / 16;
    P.heads = 1;
    P.width = P.heads * P.chunks;
    P.rows = kMoveThreads / P.width;
    P.parts = 2 * ((cache->heads + P.heads - 1) / P.heads);
    const int64_t groups = (int64_t)B * cache->layers * P.parts;
    if (groups > kMostGroups || B > kMostGroups / 4) return MDSD_E_SHAPE;
    P.by_layer = Divisor::of(cache->layers);
    P.by_part = Divisor::of(P.parts);
    P.by_width = Divisor::of(P.width);
    P.by_chunks = Divisor::of(P.chunks);
    hipStream_t st = (hipStream_t)stream;
    (void)hipGetLastError();
    hipLaunchKernelGGL(kv_select_kernel, dim3((unsigned)B), dim3(kSelectThreads), 0, st, P);
    if (hipGetLastError() != hipSuccess) return MDSD_E_LAUNCH;
    hipLaunchKernelGGL(scales ? kv_move_kernel<true> : kv_move_kernel<false>, dim3((unsigned)groups), dim3(kMoveThreads), 0, st, P);
    return hipGetLastError() == hipSuccess ? MDSD_OK : MDSD_E_LAUNCH;
}
