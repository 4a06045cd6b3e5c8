// Kernels of attention over pages of 4-bit numbers; attention.hip has the entry points.
#include "attention_mx.hpp"
#include "attention_mx_kernel.hpp"

namespace preft {

void launch_mx_attention(const AttnArgs &a, int elem, int head_dim, bool direct, dim3 grid, hipStream_t st)
{
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
    if (elem == 2) {
        if (head_dim == 128) direct ? launch(attention_mx_kernel<__bf16, 128, true>) : launch(attention_mx_kernel<__bf16, 128, false>);
        else direct ? launch(attention_mx_kernel<__bf16, 64, true>) : launch(attention_mx_kernel<__bf16, 64, false>);
    } else {
        if (head_dim == 128) direct ? launch(attention_mx_kernel<float, 128, true>) : launch(attention_mx_kernel<float, 128, false>);
        else direct ? launch(attention_mx_kernel<float, 64, true>) : launch(attention_mx_kernel<float, 64, false>);
    }
}

}  // namespace preft
