// The kernels over pages of 4-bit numbers are a translation unit of their own (attention_mx.hip).
#pragma once
#include "attention_kernel.hpp"
#include "mx4.hpp"

namespace preft {

// elem: bytes of an element of q and out
void launch_mx_attention(const AttnArgs &a, int elem, int head_dim, bool direct, dim3 grid, hipStream_t st);

}  // namespace preft
