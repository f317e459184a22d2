// How a tree attention is cut into launches, and the launchers (one source file for each element type and size of heads).
#pragma once
#include "tree_attention.h"

namespace mdsd {

struct AttentionPlan {
    int tile_rows;          // 16, 32: the narrow kernel; 64, 128: the wide one
    int slice;              // of the narrow kernel: keys of a wave in each tile
    int64_t rows, units;    // rows of a tree; units of the launch
    int row_tiles, groups;  // groups = 0: a workgroup per unit, and nothing else
    int part_rows;          // rows that a part of a unit has room for in the workspace
    int first_round;        // trees that begin first, where they go by length; 0: they go in their order
    int joint_tiles;        // 0: the shared prefix is not met by all rows together
    size_t sums, stats, ends, joint_sums, joint_stats, joint_ends, bytes;  // offsets in the workspace; 0 bytes: none
};

int attend_fp32(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st);
int attend_bf16(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st);
int attend_fp16(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st);

}  // namespace mdsd
