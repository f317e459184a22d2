// Joining the parts of rows whose keys were shared out.
#pragma once
#include "tree_attention.h"

namespace mdsd {

// Joins the parts of a unit's rows, and those of the shared prefix: with M the largest shift,
// out = sum 2^(shift_i - M) o_i / sum 2^(shift_i - M) sum_i.
struct CombineParams {
    Cache cache;
    Trees trees;
    Heads out;
    int group, rows, row_tiles;  // rows of a tile
    Divisor by_group;
    int32_t* flags;
    const int32_t* ends;
    const float* sums;
    const float2* stats;
    // of the joint launch; joint_ends = NULL: there was none
    int joint_tiles;
    const int32_t* joint_ends;
    const float* joint_sums;
    const float2* joint_stats;
};

// kLanes: of a row, four elements each
template <class T, int kLanes>
__global__ __launch_bounds__(256) void attention_combine_kernel(CombineParams P, int rows_of_group)
{
    const Cache& C = P.cache;
    const int b = blockIdx.y / C.heads, kv_head = blockIdx.y - b * C.heads;
    const int length = C.lengths[b], rows = P.trees.count(b) * P.group;
    if (length < 0) {
        if (P.flags && threadIdx.x == 0 && kv_head == 0 && blockIdx.x == 0) atomicOr(&P.flags[b], MDSD_FLAG_NO_PAGE);
        return;
    }
    const int x = threadIdx.x % kLanes * 4;
    for (int i = threadIdx.x / kLanes; i < rows_of_group; i += 256 / kLanes) {
        const int row = (int)blockIdx.x * rows_of_group + i;
        if (row >= rows || x >= C.dim) return;
        const int tile = row / P.rows;
        const int unit = (kv_head * P.trees.B + b) * P.row_tiles + tile;
        const int from = P.ends[2 * unit], to = P.ends[2 * unit + 1];
        if (from == to && !P.joint_ends) continue;  // in one part: it is done
        const int64_t own = ((int64_t)unit + from) * P.rows + row - tile * P.rows;
        int64_t joint = 0;
        int joint_parts = 0;
        if (P.joint_ends) {
            const int all = b * P.trees.N * P.group + row, joint_unit = kv_head * P.joint_tiles + all / kJointRows;
            const int first = P.joint_ends[2 * joint_unit];
            joint = ((int64_t)joint_unit + first) * kJointRows + all % kJointRows;
            joint_parts = P.joint_ends[2 * joint_unit + 1] - first + 1;
        }
        const int parts = to - from + 1;
        float most = -INFINITY;
        for (int p = 0; p < parts; ++p) most = fmaxf(most, P.stats[own + (int64_t)p * P.rows].x);
        for (int p = 0; p < joint_parts; ++p) most = fmaxf(most, P.joint_stats[joint + (int64_t)p * kJointRows].x);
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
        auto add = [&](float2 stat, f32x4 part) {
            const float factor = stat.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stat.x - most);
            sum += stat.y * factor;
            o += part * factor;
        };
#pragma unroll 4
        for (int p = 0; p < parts; ++p) {
            const int64_t at = own + (int64_t)p * P.rows;
            add(P.stats[at], *(const f32x4*)(P.sums + at * C.dim + x));
        }
#pragma unroll 4
        for (int p = 0; p < joint_parts; ++p) {
            const int64_t at = joint + (int64_t)p * kJointRows;
            add(P.joint_stats[at], *(const f32x4*)(P.joint_sums + at * C.dim + x));
        }
        o *= sum == 0.f ? 0.f : 1.f / sum;
        const int node = P.by_group(row), head = kv_head * P.group + row - node * P.group;
        char* const out = P.out.p + b * P.out.ld_tree + node * P.out.ld_node + head * P.out.ld_head;
        write_four<T>(out, x, o);
    }
}

}  // namespace mdsd
