#include "linear_attention_pass.h"

template hipError_t bagel_launch_attention_pass(const bagel_attention_pass<_Float16> &, hipStream_t);
