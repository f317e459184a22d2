#include "tree_attention_launch.h"

namespace mdsd {

int attend_fp16(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    if (dim <= 64) return attend<_Float16, 64, false>(P, plan, ws, st);
    if (dim <= 128) return attend<_Float16, 128, false>(P, plan, ws, st);
    return attend<_Float16, 256, false>(P, plan, ws, st);
}

}  // namespace mdsd
