#include "tree_attention_launch.h"

namespace mdsd {

int attend_bf16(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    return P.lse ? attend<__bf16, false, true>(dim, P, plan, ws, st) : attend<__bf16, false, false>(dim, P, plan, ws, st);
}

}  // namespace mdsd
