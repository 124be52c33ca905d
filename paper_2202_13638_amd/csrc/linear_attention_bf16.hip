// The passes of linear attention in one of the three types.
#include "linear_attention_pass.h"

template hipError_t bagel_launch_attention_memories(const bagel_attention_pass<__bf16> *, int, hipStream_t);
template hipError_t bagel_launch_attention_pass(const bagel_attention_pass<__bf16> &, hipStream_t);
template hipError_t bagel_launch_attention_keys(const bagel_attention_pass<__bf16> &, const bagel_attention_pass<__bf16> &, hipStream_t);
