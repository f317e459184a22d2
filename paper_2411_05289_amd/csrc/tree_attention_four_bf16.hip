#include "tree_attention_launch.h"

namespace mdsd {

int attend_four_bf16(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    return attend<__bf16, true, true>(dim, P, plan, ws, st);
}

}  // namespace mdsd
