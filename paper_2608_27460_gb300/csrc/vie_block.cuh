// vie_block.cuh - sums and maxima over the threads of a CTA, and one value
// of a matrix in either of the library's storage types.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace vie {

__device__ __forceinline__ float load_value(const float *p) { return *p; }
__device__ __forceinline__ float load_value(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_value(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_value(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}

// The sum / maximum of v over the NT threads of the CTA, in all of them, in
// an order that depends on NT alone.  `scratch`: 32 floats of shared memory;
// every thread of the CTA calls, and may call again at once.
template <int NT>
__device__ __forceinline__ float block_sum(float v, float *scratch) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_sum(v);
    __syncthreads();  // the last call's reads
    if (lane == 0) scratch[warp] = v;
    __syncthreads();
    return warp_sum(lane < NT / 32 ? scratch[lane] : 0.0f);
}
template <int NT>
__device__ __forceinline__ float block_max(float v, float *scratch) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_max(v);
    __syncthreads();  // the last call's reads
    if (lane == 0) scratch[warp] = v;
    __syncthreads();
    return warp_max(lane < NT / 32 ? scratch[lane] : -INFINITY);
}

}  // namespace vie
