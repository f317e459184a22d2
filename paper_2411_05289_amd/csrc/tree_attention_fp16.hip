#include "tree_attention_launch.h"

namespace mdsd {

int attend_fp16(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    return P.lse ? attend<_Float16, false, true>(dim, P, plan, ws, st) : attend<_Float16, false, false>(dim, P, plan, ws, st);
}

}  // namespace mdsd
