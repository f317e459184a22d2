#include "tree_attention_launch.h"

namespace mdsd {

int attend_fp32(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    return P.lse ? attend<float, false, true>(dim, P, plan, ws, st) : attend<float, false, false>(dim, P, plan, ws, st);
}

}  // namespace mdsd
