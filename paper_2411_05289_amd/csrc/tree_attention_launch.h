// The launches of a tree attention in one element type.
#pragma once
#include <type_traits>

#include "tree_attention_combine.h"
#include "tree_attention_narrow.h"
#include "tree_attention_plan.h"
#include "tree_attention_wide.h"

namespace mdsd {

template <class Kernel>
static int launch_attention(Kernel kernel, const AttentionParams& P, int64_t groups, size_t lds, hipStream_t st)
{
    if (!P.trees.complete) lds += P.trees.N * sizeof(int);
    if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
        return MDSD_E_LAUNCH;
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(kAttentionThreads), lds, st, P);
    return hipGetLastError() == hipSuccess ? MDSD_OK : MDSD_E_LAUNCH;
}

// kSums: the rows' sums may be asked for; in 4 bits builds without them are left out
template <class T, int kDim, bool kFour, bool kSums>
static int attend(AttentionParams P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    (void)hipGetLastError();
    P.row_tiles = plan.row_tiles;
    P.by_tiles = Divisor::of(plan.row_tiles);
    P.groups = plan.groups;
    P.part_rows = plan.part_rows;
    P.first_round = plan.first_round;
    if (plan.groups) {
        P.ends = (int32_t*)(ws + plan.ends);
        P.sums = (float*)(ws + plan.sums);
        P.stats = (float2*)(ws + plan.stats);
    }
    if (plan.joint_tiles) {
        P.joint_tiles = plan.joint_tiles;
        P.joint_ends = (int32_t*)(ws + plan.joint_ends);
        P.joint_sums = (float*)(ws + plan.joint_sums);
        P.joint_stats = (float2*)(ws + plan.joint_stats);
    }
    const int64_t groups = plan.groups ? plan.groups : plan.units;
    auto either = [&](auto line, auto unit, size_t lds) {
        return plan.groups ? launch_attention(line, P, groups, lds, st) : launch_attention(unit, P, groups, lds, st);
    };
    int rc = MDSD_E_SHAPE;
    constexpr int kRowBytes = kDim * sizeof(Worked<T, kFour>);
    auto narrow = [&](auto tiles, auto slice) {
        constexpr int kTiles = decltype(tiles)::value, kSlice = decltype(slice)::value;
        constexpr size_t kLds = NarrowTile<T, kDim, kTiles, kSlice, kFour>::kLds;
        if constexpr (kTiles == 1 && ((kRowBytes == 512 && kSlice == 32) || (kRowBytes == 256 && kSlice == 16))) {  // shared out only
            return launch_attention(P.cache.dim == kDim ? attention_narrow_kernel<T, kDim, kTiles, kSlice, true, true, kFour, kSums>
                                                        : attention_narrow_kernel<T, kDim, kTiles, kSlice, true, false, kFour, kSums>,
                                    P, groups, kLds, st);
        } else {
            return P.cache.dim == kDim ? either(attention_narrow_kernel<T, kDim, kTiles, kSlice, true, true, kFour, kSums>,
                                                attention_narrow_kernel<T, kDim, kTiles, kSlice, false, true, kFour, kSums>, kLds)
                                       : either(attention_narrow_kernel<T, kDim, kTiles, kSlice, true, false, kFour, kSums>,
                                                attention_narrow_kernel<T, kDim, kTiles, kSlice, false, false, kFour, kSums>, kLds);
        }
    };
    using one = std::integral_constant<int, 1>;
    using two = std::integral_constant<int, 2>;
    using few = std::integral_constant<int, 16>;
    using many = std::integral_constant<int, 32>;
    if (plan.joint_tiles)
        rc = launch_attention(attention_wide_kernel<T, kDim, 4, true, true, kFour, false>, P, groups, WideTile<T, kDim, 4, kFour>::kLds, st);
    else if (plan.tile_rows == 128)
        rc = either(attention_wide_kernel<T, kDim, 4, true, false, kFour, kSums>, attention_wide_kernel<T, kDim, 4, false, false, kFour, kSums>, WideTile<T, kDim, 4, kFour>::kLds);
    if constexpr (kRowBytes >= 256)
        if (plan.slice == 16) rc = narrow(one(), few());
    if constexpr (kRowBytes <= 256 || kRowBytes == 2 * kDim)
        if (plan.tile_rows == 16 && plan.slice == 32) rc = narrow(one(), many());
    if constexpr (kDim <= 128)
        if (plan.tile_rows == 32) rc = narrow(two(), many());
    if constexpr (kRowBytes <= 512)
        if (plan.tile_rows == 64)
            rc = either(attention_wide_kernel<T, kDim, 2, true, false, kFour, kSums>, attention_wide_kernel<T, kDim, 2, false, false, kFour, kSums>, WideTile<T, kDim, 2, kFour>::kLds);
    if (rc != MDSD_OK || !plan.groups) return rc;
    CombineParams C = {};
    C.cache = P.cache;
    C.trees = P.trees;
    C.out = P.out;
    C.group = P.group;
    C.rows = plan.tile_rows;
    C.row_tiles = plan.row_tiles;
    C.part_rows = plan.part_rows;
    C.by_group = P.by_group;
    C.scale = P.scale;
    C.flags = P.flags;
    C.ends = P.ends;
    C.sums = P.sums;
    C.stats = P.stats;
    C.joint_tiles = P.joint_tiles;
    C.shared = P.shared;
    C.joint_ends = P.joint_ends;
    C.joint_sums = P.joint_sums;
    C.joint_stats = P.joint_stats;
    C.lse = P.lse;
    C.by_unit = P.by_unit;
    // as many lanes to a row as its parts keep busy (a workgroup's rows divide a tile's: they are of one unit)
    const int stands = 1024 / kDim;
    int slices = 1;
    while (slices < stands && slices * 4 * plan.units < plan.groups) slices *= 2;
    const int rows_of_group = stands / slices;
    hipLaunchKernelGGL((attention_combine_kernel<T, kDim / 4, kFour, kSums>),
                       dim3((unsigned)(P.trees.B * P.cache.heads), (unsigned)((plan.rows + rows_of_group - 1) / rows_of_group)),
                       dim3(kAttentionThreads), 0, st, C, slices);
    return hipGetLastError() == hipSuccess ? MDSD_OK : MDSD_E_LAUNCH;
}

template <class T, bool kFour, bool kSums>
static int attend(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    if (dim <= 64) return attend<T, 64, kFour, kSums>(P, plan, ws, st);
    if (dim <= 128) return attend<T, 128, kFour, kSums>(P, plan, ws, st);
    return attend<T, 256, kFour, kSums>(P, plan, ws, st);
}

}  // namespace mdsd
