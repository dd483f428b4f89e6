// What the row kernels (layer norm, bias + GELU, distillation) share: elements of both types as fp32, sums over a workgroup.
#pragma once
#include "tmask_device.hpp"

namespace tmask {

// element i of an array of type DT, as fp32
template <int DT>
__device__ __forceinline__ float load_one(const void *p, size_t i)
{
    if constexpr (DT == kF32)
        return ((const float *)p)[i];
    else
        return __uint_as_float((uint32_t)((const uint16_t *)p)[i] << 16);
}

// rounded to nearest even
template <int DT>
__device__ __forceinline__ void store_one(void *p, size_t i, float v)
{
    if constexpr (DT == kF32)
        ((float *)p)[i] = v;
    else
        ((__bf16 *)p)[i] = (__bf16)v;
}

// sum over the workgroup, in every thread; `red` has a place for each wavefront and may be used again at once
template <int WAVES>
__device__ __forceinline__ float group_sum(float v, float *red)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        v += __shfl_xor(v, d, 64);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0)
            red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; w++)
            v += red[w];
        __syncthreads();
    }
    return v;
}

template <int WAVES>
__device__ __forceinline__ float group_max(float v, float *red)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        v = fmaxf(v, __shfl_xor(v, d, 64));
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0)
            red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < WAVES; w++)
            v = fmaxf(v, red[w]);
        __syncthreads();
    }
    return v;
}

}  // namespace tmask
