// The scan that the one-workgroup schedule kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace preft {

constexpr int SCHED_THREADS = 1024;

// Exclusive scan of one int per thread over the block; returns the block total through *total.  Sums past 31 bits, which only malformed tables give, wrap.
__device__ __forceinline__ int32_t block_exclusive_scan(int32_t v, int32_t *lds /* >= 32 ints */, int32_t *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6;
    uint32_t incl = (uint32_t)v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t up = __shfl_up(incl, off, 64);
        if (lane >= off) incl += up;
    }
    if (n_waves == 1) {                      // uniform
        __syncthreads();                     // as below: what the wavefront did to LDS before a scan is seen after it
        *total = (int32_t)__shfl(incl, 63, 64);
        return (int32_t)(incl - (uint32_t)v);
    }
    __syncthreads();                         // lds may still be read from a previous scan
    if (lane == 63) lds[wave] = (int32_t)incl;
    __syncthreads();
    uint32_t base = 0, sum = 0;
    for (int w = 0; w < n_waves; ++w) {
        const uint32_t t = (uint32_t)lds[w];
        if (w < wave) base += t;
        sum += t;
    }
    *total = (int32_t)sum;
    return (int32_t)(base + incl - (uint32_t)v);
}

}  // namespace preft
