#include "tree_attention_launch.h"

namespace mdsd {

int attend_fp32(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    if (dim <= 64) return attend<float, 64, false>(P, plan, ws, st);
    if (dim <= 128) return attend<float, 128, false>(P, plan, ws, st);
    return attend<float, 256, false>(P, plan, ws, st);
}

}  // namespace mdsd
