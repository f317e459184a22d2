// Joining the parts of rows whose keys were shared out.
#pragma once
#include "tree_attention.h"

namespace mdsd {

// Joins the parts of a unit's rows, and those of the shared prefix: with f_i from part i's score to the largest of them
// (rebased), out = sum f_i o_i / sum f_i sum_i.  Bound by its few loads, one behind the other, and the launch: 4.3 us
// for a token's 256 parts, 18 us for 64 MB of a shared prefix's (grouping rows otherwise changed nothing).
struct CombineParams {
    Cache cache;
    Trees trees;
    Heads out;
    int group, rows, row_tiles, part_rows;  // rows of a tile; that a part has room for
    Divisor by_group;
    float scale;
    int32_t* flags;
    const int32_t* ends;
    const float* sums;
    const float2* stats;
    float* lse;
    // of the joint launch; joint_ends = NULL: there was none
    int joint_tiles, shared;
    const int32_t* joint_ends;
    const float* joint_sums;
    const float2* joint_stats;
    bool by_unit;
};

// kLanes: of a row, four elements each; they first stand for a part each, whose factor they form.  `slices` rows of lanes
// share a row's parts (units whose keys went to many workgroups).
template <class T, int kLanes, bool kFour, bool kSums>
__global__ __launch_bounds__(kAttentionThreads) void attention_combine_kernel(CombineParams P, int slices)
{
    __shared__ f32x4 sums_of[kAttentionThreads];
    const Cache& C = P.cache;
    const int b = blockIdx.x / C.heads, kv_head = blockIdx.x - b * C.heads;
    const int rows_here = kAttentionThreads / kLanes / slices, first_row = (int)blockIdx.y * rows_here;
    // (a tile's rows lie in one workgroup's: one unit; a tree without rows or own slots may have none, and what stands there is
    // not used)
    const int tile = first_row / P.rows, unit = kFour && P.by_unit ? (b * P.row_tiles + tile) * C.heads + kv_head : (kv_head * P.trees.B + b) * P.row_tiles + tile;
    const int from = P.ends[2 * unit], last = P.ends[2 * unit + 1];
    const int length = C.lengths[b], rows = P.trees.count(b) * P.group, capacity = C.table_pages * C.page_size;
    if (length < 0) {
        if (P.flags && threadIdx.x == 0 && kv_head == 0 && blockIdx.y == 0) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
        return;
    }
    const int lane = threadIdx.x % kLanes, x = lane * 4, stand = threadIdx.x / kLanes, slice = stand % slices;
    const int column = min(x, C.dim - 4), row = first_row + stand / slices;
    const bool valid = row < rows;
    const bool own_slots = first_own_slot(P.joint_ends != nullptr, P.shared, length, capacity) < capacity;
    const int parts = own_slots ? last - from + 1 : 0;
    if (first_row >= rows || (parts == 1 && !P.joint_ends)) return;  // nothing there; it is done
    // (no unit is there to say that the nodes' slots have no page)
    if (!own_slots && P.flags && threadIdx.x == 0 && kv_head == 0 && blockIdx.y == 0) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
    // the row's parts: those of its tree's unit, and those of the shared prefix
    struct Parts {
        const float* sums;
        const float2* stats;
        int number, rows;
    } of[2] = {{nullptr, nullptr, 0, 0}, {nullptr, nullptr, 0, 0}};
    if (valid && own_slots) {
        const int64_t own = ((int64_t)unit + from) * P.part_rows + row - tile * P.rows;
        of[0] = {P.sums + own * C.dim, P.stats + own, parts, P.part_rows};
    }
    if (valid && P.joint_ends) {
        const int all = b * P.trees.N * P.group + row, joint_unit = kv_head * P.joint_tiles + all / kJointRows;
        const int first = P.joint_ends[2 * joint_unit];
        const int64_t joint = ((int64_t)joint_unit + first) * kJointRows + all % kJointRows;
        of[1] = {P.joint_sums + joint * C.dim, P.joint_stats + joint, P.joint_ends[2 * joint_unit + 1] - first + 1, kJointRows};
    }
    // the first parts' statistics and sums are asked for together
    float2 stat[2];
    f32x4 part[4];
#pragma unroll
    for (int w = 0; w < 2; ++w)
        stat[w] = lane < of[w].number ? of[w].stats[(int64_t)lane * of[w].rows] : float2{-INFINITY, 0.f};
    auto load_parts = [&](const Parts& from, int p0, int p, int here) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            part[j] = *(const f32x4*)(from.sums + (int64_t)(p0 + min(p + j * slices, here - 1)) * from.rows * C.dim + column);
    };
    if (of[0].number) load_parts(of[0], 0, slice, min(kLanes, of[0].number));
    float most = fmaxf(stat[0].x, stat[1].x);
#pragma unroll
    for (int w = 0; w < 2; ++w)
        for (int p = lane + kLanes; p < of[w].number; p += kLanes) most = fmaxf(most, of[w].stats[(int64_t)p * of[w].rows].x);
#pragma unroll
    for (int d = kLanes / 2; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        for (int p0 = 0; p0 < of[w].number; p0 += kLanes) {
            const int mine = p0 + lane, here = min(kLanes, of[w].number - p0);
            if (p0) stat[w] = mine < of[w].number ? of[w].stats[(int64_t)mine * of[w].rows] : float2{-INFINITY, 0.f};
            const float factor = rebased<T>(stat[w].x, most, P.scale);
            sum += stat[w].y * factor;
            for (int p = slice; p < here; p += 4 * slices) {
                if (w || p0 || p != slice) load_parts(of[w], p0, p, here);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float of_part = __shfl(factor, min(p + j * slices, here - 1), kLanes);
                    if (p + j * slices < here) o += part[j] * of_part;
                }
            }
        }
    }
#pragma unroll
    for (int d = kLanes / 2; d; d >>= 1) sum += __shfl_xor(sum, d);
    if (slices > 1) {
        sums_of[threadIdx.x] = o;
        __syncthreads();
        if (slice == 0)
            for (int w = 1; w < slices; ++w) o += sums_of[threadIdx.x + w * kLanes];
    }
    if (valid && slice == 0 && x < C.dim) {
        o *= sum == 0.f ? 0.f : 1.f / sum;
        const int node = P.by_group(row), head = kv_head * P.group + row - node * P.group;
        if (kSums && P.lse && lane == 0) P.lse[((int64_t)b * P.trees.N + node) * (C.heads * P.group) + head] = log_of_sum<T>(most, sum, P.scale);
        write_four<T>(P.out.p + b * P.out.ld_tree + node * P.out.ld_node + head * P.out.ld_head, x, o);
    }
}

}  // namespace mdsd
