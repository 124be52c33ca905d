// The passes of linear attention in one of the three types.
#include "linear_attention_pass.h"

template hipError_t bagel_launch_attention_memories(const bagel_attention_pass<float> *, int, hipStream_t);
template hipError_t bagel_launch_attention_pass(const bagel_attention_pass<float> &, hipStream_t);
