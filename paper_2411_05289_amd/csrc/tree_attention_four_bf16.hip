#include "tree_attention_launch.h"

namespace mdsd {

int attend_four_bf16(int dim, const AttentionParams& P, const AttentionPlan& plan, char* ws, hipStream_t st)
{
    if (dim <= 64) return attend<__bf16, 64, true>(P, plan, ws, st);
    if (dim <= 128) return attend<__bf16, 128, true>(P, plan, ws, st);
    return attend<__bf16, 256, true>(P, plan, ws, st);
}

}  // namespace mdsd
