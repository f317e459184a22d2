#include "tree_attention_launch.h"

namespace mdsd {

int attend_four_fp32(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    return attend<float, true, true>(dim, P, plan, ws, st);
}

}  // namespace mdsd
