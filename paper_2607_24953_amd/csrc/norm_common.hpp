// Device-side helpers of the norm kernels (gfx950 only).
#pragma once

#include "device_common.hpp"

namespace q2d {

// element i of a float32 or bfloat16 array
__device__ __forceinline__ float load_value(const void *p, int bf16, int64_t i)
{
    return bf16 ? bf16_to_f(reinterpret_cast<const uint16_t *>(p)[i]) : reinterpret_cast<const float *>(p)[i];
}
__device__ __forceinline__ void store_value(void *p, int bf16, int64_t i, float v)
{
    if (bf16) reinterpret_cast<uint16_t *>(p)[i] = f_to_bf16_rne(v);
    else reinterpret_cast<float *>(p)[i] = v;
}

// Sum over a workgroup of `waves` waves, the same value in every lane; `lds` holds one
// double a wave.  The order of the additions is fixed.
__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ double group_sum(double v, int waves, double *lds)
{
    v = wave_sum(v);
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    for (int i = 0; i < waves; ++i) s += lds[i];
    __syncthreads();
    return s;
}

// 1 / sqrt(mean + eps), rounded to float32 once
__device__ __forceinline__ float rstd_of(double sum, int64_t cols, double eps)
{
    return (float)(1.0 / __builtin_sqrt(sum / (double)cols + eps));
}

}  // namespace q2d
