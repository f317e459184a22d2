#include "tree_attention_launch.h"

namespace mdsd {

int attend_fp32(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    if (dim <= 64) return attend<float, 64>(P, plan, ws, st);
    if (dim <= 128) return attend<float, 128>(P, plan, ws, st);
    return attend<float, 256>(P, plan, ws, st);
}

}  // namespace mdsd
