#include "tree_attention_launch.h"

namespace mdsd {

int attend_four_fp32(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    if (dim <= 64) return attend<float, 64, true>(P, plan, ws, st);
    if (dim <= 128) return attend<float, 128, true>(P, plan, ws, st);
    return attend<float, 256, true>(P, plan, ws, st);
}

}  // namespace mdsd
