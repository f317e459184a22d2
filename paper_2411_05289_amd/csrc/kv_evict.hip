// Sequences cut to the slots that matter: which those are, and their way to the front.
//
// Two launches.  `select`: a workgroup per sequence finds the weight of the last slot that is kept by its digits, the highest
// first (three counts of 11, 11 and 10 bits), and then goes through the slots once, in order, giving each that is kept its
// new place.  `move`: what is kept only moves to the front, so that a workgroup that reads some rows in a row before it
// writes them overwrites nothing that is read later; it has some chunks of keys or values in one layer to itself.
//
// Measured: 32 sequences of 1000 to 8192 slots cut to 2048, 8 layers of 8 heads of 128 in 4 bits, 935 MB in 245 us, 3.8 TB/s (a kept row
// of 64 bytes brings a line of 128 with it: 5 TB/s of lines), and 11 us of selection; one of 16500 cut to 4096, 4 layers in bf16,
// 134 MB in 40 us by 256 workgroups, and 18 us of selection by one.
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
    int held;         // of a selection: weights that there is room for
    int chunks;       // of 16 bytes, of a head
    int width, rows;  // of a move's workgroup: chunks, rows that its threads have at once
    Divisor by_layer, by_part, by_width, by_chunks;
    int parts;  // of a layer: of keys and of values in turn
    bool halves;  // of a part, are each a workgroup's
    int groups;   // of whole parts
};

constexpr uint32_t kAlways = 0xffffffffu;  // the rank of slots that are kept whatever their weight is, and of no number
constexpr int kSelectThreads = 1024, kDigits = 2048, kEach = 4, kSelectAhead = 4, kMoveThreads = 256, kLookThreads = 256, kMoveAhead = 8, kMoveRows = 64, kMostHeld = 32768;

// Whole numbers in the weights' order; NaN is the least, and the zeros are one
__device__ inline uint32_t rank_of(float x)
{
    const uint32_t bits = __float_as_uint(x + 0.f);
    return x != x ? 0 : bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u);
}

// Bits of the lanes before this one
__device__ inline int bits_below(uint64_t x)
{
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(x >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)x, 0));
}

// Sum over the threads before this one, and over all; `sums`: one for each wave (barriers inside)
__device__ inline int sum_before(int x, int* sums, int* all)
{
    const int wave = threadIdx.x >> 6, up = sum_up_to(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sums[wave] = up;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kSelectThreads / 64; ++w) {
        const int of = sums[w];
        before += w < wave ? of : 0;
        total += of;
    }
    *all = total;
    return before + up - x;
}

// A barrier that waits for LDS alone, and for no load or store of memory
__device__ inline void meet_in_lds()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Sequences of up to P.held slots have their weights in LDS, read from memory once, and counted by their first digit on the way.
// kHeld: all do.  As a launch has one turn of everything, the code's own way from memory counts: 4 slots a thread at a time, not 8, and
// a build without what longer sequences need take 4 us of 15 from four sequences of 100 to 200 slots.  (The other, four layers, with moving:
// one sequence of 40000 slots cut to 4096 91 us, where one of 30000 takes 66; one of 131072 in 4 bits cut to 16384 272.)
template <bool kHeld>
__global__ __launch_bounds__(kSelectThreads) void kv_select_kernel(EvictParams P)
{
    extern __shared__ float in_lds[];
    __shared__ int counts[kDigits], sums[kSelectThreads / 64], stretch[2][kSelectThreads / 64];
    __shared__ uint32_t chosen;
    __shared__ int chosen_left, chosen_all;
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
    const bool held = kHeld || length <= P.held;
    auto rank_with = [&](int s, float w) { return s >= P.first && s < last ? rank_of(w) : kAlways; };
    if (held) {
        for (int i = threadIdx.x; i < kDigits; i += kSelectThreads) counts[i] = 0;
        // (all of them asked for at once, and 4096 slots at a time only if there are)
        constexpr int kStretches = kMostHeld / (kSelectThreads * kEach);
        float w[kStretches][kEach];
        const int there = min(length, P.slots);
#pragma unroll
        for (int i = 0; i < kStretches; ++i)
            if (i * kSelectThreads * kEach < length) {
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    const int s = (i * kEach + j) * kSelectThreads + threadIdx.x;
                    w[i][j] = weights[min(s, there - 1)];
                }
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kStretches; ++i)
            if (i * kSelectThreads * kEach < length) {
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    const int s = (i * kEach + j) * kSelectThreads + threadIdx.x;
                    if (s >= there) w[i][j] = 0.f;
                    if (s < length) in_lds[s] = w[i][j];
                    if (s >= P.first && s < last) atomicAdd(&counts[rank_of(w[i][j]) >> 21], 1);
                }
            }
        __syncthreads();
    }
    auto weight_at = [&](int s) { return held ? in_lds[s] : weight_of(s); };
    int left = P.budget - P.first - P.recent;
    uint32_t border = 0;  // ranks above it are kept, and `left` of those that are it
    if (left > 0) {
        uint32_t known = 0;
        for (int shift = 21; shift >= 0; shift = shift ? (shift == 21 ? 10 : 0) : -1) {
            const int bits = shift ? 11 : 10;
            const bool counted = held && shift == 21;
            if (!counted) {
                for (int i = threadIdx.x; i < kDigits; i += kSelectThreads) counts[i] = 0;
                __syncthreads();
            }
            for (int s0 = P.first + threadIdx.x; !counted && s0 < last; s0 += kSelectThreads * kSelectAhead) {
                const int here = (last - (s0 - (int)threadIdx.x) + kSelectThreads - 1) / kSelectThreads;  // of all threads together
                uint32_t rank[kSelectAhead];
#pragma unroll
                for (int j = 0; j < kSelectAhead; ++j)
                    if (j < here) rank[j] = rank_of(weight_at(min(s0 + j * kSelectThreads, last - 1)));
#pragma unroll
                for (int j = 0; j < kSelectAhead; ++j) {
                    const uint32_t r = rank[j];
                    if (j < here && s0 + j * kSelectThreads < last && ((r ^ border) & known) == 0) atomicAdd(&counts[r >> shift & ((1 << bits) - 1)], 1);
                }
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
                chosen_all = chosen_left == (upper ? n0 : n1);
            }
            __syncthreads();
            border |= chosen << shift;
            known |= (uint32_t)((1 << bits) - 1) << shift;
            left = chosen_left;
            if (chosen_all && border) {  // all that begin like this are kept: whatever is above the rank in front of them
                border -= 1;
                left = 0;
                break;
            }
            __syncthreads();
        }
    }
    // The places of what is kept: of those at the border the first `left` (none, where only the first and the last are kept:
    // `border` is then no slot's rank).  A wave has kEach times 64 slots in a row, and a bit for each.
    if (P.budget == P.first + P.recent) border = kAlways - 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int number = 0, equal = 0;  // kept above the border, and at it, so far
    for (int from = 0; from < length; from += kSelectThreads * kEach) {
        const int s0 = from + wave * 64 * kEach + lane;
        uint64_t above[kEach], at_border[kEach];
        float w[kEach];
        int counted = 0;  // (both in one: there are below 2^15 of a kind at a time)
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int s = min(s0 + j * 64, length - 1);
            w[j] = weight_at(s);
            const uint32_t r = rank_with(s, w[j]);
            above[j] = __ballot(r > border);
            at_border[j] = __ballot(r == border);
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int there = length - (from + wave * 64 * kEach + j * 64);
            const uint64_t slots = there >= 64 ? ~0ull : there > 0 ? (1ull << there) - 1 : 0;
            above[j] &= slots;
            at_border[j] &= slots;
            counted += __popcll(above[j]) | __popcll(at_border[j]) << 16;
        }
        // (sums in two places in turn, so that one barrier is enough; in memory weights have to be there before others' are written over them)
        int* const sum = stretch[from / (kSelectThreads * kEach) & 1];
        if (lane == 0) sum[wave] = counted;
        if (held)
            meet_in_lds();
        else
            __syncthreads();
        // (a lane for each wave)
        const int of = lane < kSelectThreads / 64 ? sum[lane] : 0, up_to = sum_up_to(of);
        const int before = __builtin_amdgcn_readlane(up_to, wave) - counted, all = __builtin_amdgcn_readlane(up_to, kSelectThreads / 64 - 1);
        int n = number + (before & 0xffff), e = equal + (before >> 16);
        number += all & 0xffff;
        equal += all >> 16;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int e_here = e + bits_below(at_border[j]), at = n + bits_below(above[j]) + min(e_here, left);
            if ((above[j] | (e_here < left ? at_border[j] : 0)) >> lane & 1) {
                kept[at] = s0 + j * 64;
                // (every thread has its weights by now, and what comes later stands behind all of these places)
                if (out && at < P.slots) out[at] = w[j];
            }
            n += __popcll(above[j]);
            e += __popcll(at_border[j]);
        }
    }
    __syncthreads();
    if (out)
        for (int s = P.budget + threadIdx.x; s < P.slots; s += kSelectThreads) out[s] = 0.f;
}

// Of a move: `width` chunks of a row (of a head, a part of one, or several) by kMoveAhead rows a thread.  Four waves move, two
// batches of rows asked for before one is written; four more look up the places of rows further on, as in one wave these loads would
// wait for the rows', and the rows for these.
template <bool kFour>
__global__ __launch_bounds__(kMoveThreads + kLookThreads) void kv_move_kernel(EvictParams P)
{
    constexpr int kBatch = kMoveRows * kMoveAhead, kLooked = kBatch / kLookThreads;
    constexpr int kTurns = 5;  // a batch that is written, three ahead of it, and one that some threads may still write
    __shared__ int64_t from[kTurns][kBatch], to[kTurns][kBatch];  // places of batches in turn; to -1: nothing moves, and any place is read
    const Cache& C = P.cache;
    // (parts in another order in each layer, as one order puts the same heads of all layers on an XCD: one sequence, 4 layers, 69 us, 67)
    // (the halves of a part eight workgroups from each other: in one XCD, whose L2 has the other half of the lines already)
    const int at_group = (int)blockIdx.x, half = P.halves ? at_group >> 3 & 1 : 0, group = P.halves ? (at_group >> 4) * 8 + (at_group & 7) : at_group;
    if (group >= P.groups) return;
    const int bl = P.by_part(group), part = (group - bl * P.parts + 2 * bl) % P.parts, b = P.by_layer(bl), layer = bl - b * C.layers;
    const int32_t* const kept = P.kept + (int64_t)b * P.budget;
    const int32_t* const table = C.table + b * C.ld_table;
    if (kept[P.budget - 1] < P.budget) return;  // nothing moves: shorter, or as long (a slot never moves up)
    // the first that moves, from lo to hi (which does): a 64th of the rest a turn, as each turn is a way to memory
    int lo = P.first, hi = P.budget - 1;
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64, at = min(lo + ((int)(threadIdx.x & 63) + 1) * step - 1, hi);
        lo += __popcll(__ballot(kept[at] == at)) * step;
        hi = min(lo + step - 1, hi);
    }
    const int batch = P.rows * kMoveAhead, batches = (P.budget - lo + batch - 1) / batch;

    if (threadIdx.x >= kMoveThreads) {
        // a lane looks up some rows of each batch: first what is kept, then its pages, then the places
        const int lane = threadIdx.x - kMoveThreads;
        int next_slot[kLooked];
        auto ask_for_slots = [&](int j) {
#pragma unroll
            for (int l = 0; l < kLooked; ++l) {
                const int i = lane + l * kLookThreads, row = lo + j * batch + i;
                next_slot[l] = i < batch && row < P.budget ? kept[row] : -1;
            }
        };
        auto look_up = [&](int j) {
            int slot[kLooked], source_page[kLooked], target_page[kLooked];
#pragma unroll
            for (int l = 0; l < kLooked; ++l) {
                const int row = lo + j * batch + lane + l * kLookThreads;
                slot[l] = next_slot[l];
                source_page[l] = target_page[l] = -1;
                if (slot[l] >= 0) {  // (the target is in front of it, and both in the table)
                    source_page[l] = table[C.by_page(slot[l])];
                    target_page[l] = table[C.by_page(row)];
                }
            }
            ask_for_slots(j + 1);
#pragma unroll
            for (int l = 0; l < kLooked; ++l) {
                const int i = lane + l * kLookThreads, row = lo + j * batch + i;
                int64_t source = -1, target = -1;
                if (slot[l] >= 0) {
                    source = place_in_page(C, source_page[l], slot[l], C.by_page(slot[l]));
                    target = place_in_page(C, target_page[l], row, C.by_page(row));
                    if (P.flags && part == 0 && layer == 0 && (source < 0 || target < 0)) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
                }
                const bool moves = source >= 0 && target >= 0;
                from[j % kTurns][i] = moves ? source : 0;
                to[j % kTurns][i] = moves ? target : -1;
            }
        };
        ask_for_slots(0);
        auto blank = [&](int j) {  // nothing is there, and nothing moves
            for (int i = lane; i < kBatch; i += kLookThreads) from[j % kTurns][i] = 0, to[j % kTurns][i] = -1;
        };
        for (int j = 0; j < 3; ++j) j < batches ? look_up(j) : blank(j);
        __syncthreads();
        for (int j = 0; j < batches; ++j) {
            j + 3 < batches ? look_up(j + 3) : blank(j + 3);
            __syncthreads();
        }
        return;
    }

    const int at_row = P.by_width((int)threadIdx.x), item = (P.halves ? (part >> 1) * 2 + half : part >> 1) * P.width + threadIdx.x - at_row * P.width;
    const int head = P.by_chunks(item);
    const bool mine = at_row < P.rows && head < C.heads;
    const int64_t column = mine ? layer * C.ld_layer + head * C.ld_head + (item - head * P.chunks) * 16 : 0;
    char* const base = (part & 1 ? C.v : C.k) + column;
    uint8_t* const scale = kFour ? (part & 1 ? P.scales.v : P.scales.k) + (column >> 4) : nullptr;
    struct Rows {
        u32x4 x[kMoveAhead];
        uint32_t y[kMoveAhead];
    } rows[3];
    const int own_row = mine ? at_row : 0;
    // (every load is made, whatever there is to move: their number tells when the oldest are there)
    auto read = [&](int j, Rows& into) {
        int64_t source[kMoveAhead];
#pragma unroll
        for (int r = 0; r < kMoveAhead; ++r) source[r] = from[j % kTurns][own_row + r * P.rows];
#pragma unroll
        for (int r = 0; r < kMoveAhead; ++r) {
            into.x[r] = *(const u32x4*)(base + source[r]);
            if (kFour) into.y[r] = scale[source[r] >> 4];
        }
    };
    __syncthreads();
    read(0, rows[0]);
    read(1, rows[1]);
    auto step = [&](int j, Rows& here, Rows& next) {
        if (j >= batches) return;
        read(j + 2, next);
        // all rows of this batch have been read before any of them is written
#pragma unroll
        for (int r = 0; r < kMoveAhead; ++r) {
            asm volatile("" : "+v"(here.x[r]));
            if (kFour) asm volatile("" : "+v"(here.y[r]));
        }
        __syncthreads();
        int64_t target[kMoveAhead];
#pragma unroll
        for (int r = 0; r < kMoveAhead; ++r) target[r] = mine ? to[j % kTurns][own_row + r * P.rows] : -1;
#pragma unroll
        for (int r = 0; r < kMoveAhead; ++r)
            if (target[r] >= 0) {
                *(u32x4*)(base + target[r]) = here.x[r];
                if (kFour) scale[target[r] >> 4] = (uint8_t)here.y[r];
            }
    };
    for (int j = 0; j < batches; j += 3) {
        step(j, rows[0], rows[2]);
        step(j + 1, rows[1], rows[0]);
        step(j + 2, rows[2], rows[1]);
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
    // A workgroup's chunks: of one head, or of several while they are fewer than eight (rows of 64 bytes, 32 sequences of 2048 slots: one head
    // 283 us, two 260, four 269); a cache line of a head where there would be few workgroups otherwise
    const int all = cache->heads * P.chunks;
    // and, where little moves, of as many as its threads have at once (18 rows of 97 sequences, 16 layers: 186 us, 46).
    P.width = P.chunks;
    while (P.width * 2 <= all && P.width * 2 <= kMoveThreads && (int64_t)P.width * 2 * (budget - first) <= kMoveThreads * kMoveAhead &&
           (int64_t)B * cache->layers * 2 * (all / (2 * P.width)) >= 1024)
        P.width *= 2;
    while (P.width * 2 <= all && P.width < 8) P.width *= 2;
    while (P.width > 8 && P.width % 2 == 0 && (int64_t)B * cache->layers * 2 * (all / P.width) < 1024) P.width /= 2;
    P.parts = 2 * ((all + P.width - 1) / P.width);
    const int64_t groups = (int64_t)B * cache->layers * P.parts;
    if (groups > kMostGroups / 2 || B > kMostGroups / 4) return MDSD_E_SHAPE;  // (of more than 256 threads)
    P.groups = (int)groups;
    // Half a line a workgroup, where whole ones leave half of the compute units empty (one sequence, 4 layers of 8 heads: 64 us, 60)
    P.halves = P.width == 8 && groups <= 128;
    if (P.halves) P.width = 4;
    P.rows = kMoveThreads / P.width < kMoveRows ? kMoveThreads / P.width : kMoveRows;
    P.by_layer = Divisor::of(cache->layers);
    P.by_part = Divisor::of(P.parts);
    P.by_width = Divisor::of(P.width);
    P.by_chunks = Divisor::of(P.chunks);
    hipStream_t st = (hipStream_t)stream;
    (void)hipGetLastError();
    const int64_t capacity = (int64_t)cache->table_pages * cache->page_size;
    P.held = (int)(capacity < kMostHeld ? capacity : kMostHeld);
    const size_t lds = (size_t)P.held * sizeof(uint32_t);
    // (the same for all calls: others may be made at once)
    const auto select = capacity <= kMostHeld ? kv_select_kernel<true> : kv_select_kernel<false>;
    if (hipFuncSetAttribute((const void*)select, hipFuncAttributeMaxDynamicSharedMemorySize, kMostHeld * (int)sizeof(uint32_t)) != hipSuccess)
        return MDSD_E_LAUNCH;
    hipLaunchKernelGGL(select, dim3((unsigned)B), dim3(kSelectThreads), lds, st, P);
    if (hipGetLastError() != hipSuccess) return MDSD_E_LAUNCH;
    hipLaunchKernelGGL(scales ? kv_move_kernel<true> : kv_move_kernel<false>, dim3((unsigned)(P.halves ? (groups + 7) / 8 * 16 : groups)), dim3(kMoveThreads + kLookThreads), 0, st, P);
    return hipGetLastError() == hipSuccess ? MDSD_OK : MDSD_E_LAUNCH;
}
