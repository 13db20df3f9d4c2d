// Device-side helpers of the norm kernels (gfx950 only).
#pragma once

#include "device_common.hpp"

namespace q2d {

typedef __bf16 bf16v2 __attribute__((ext_vector_type(2)));
typedef float f32v2 __attribute__((ext_vector_type(2)));

// two float32 values as one word of bfloat16, rounded to nearest even
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32v2{lo, hi}, bf16v2));
}
__device__ __forceinline__ float round_bf16(float v) { return bits_f(pack_bf16(v, v) << 16); }

// 16 bytes at any address of an element: the hardware takes a 16-byte access there too, in the same
// instruction, so rows need no alignment
typedef u4v u4v_any __attribute__((aligned(2)));
// (ONCE: of data that is not read or written again soon)
template <bool ONCE = false>
__device__ __forceinline__ u4v load16(const uint8_t *p)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u4v_any *>(p));
    else return *reinterpret_cast<const u4v_any *>(p);
}
template <bool ONCE = false>
__device__ __forceinline__ void store16(uint8_t *p, u4v v)
{
    if constexpr (ONCE) __builtin_nontemporal_store(v, reinterpret_cast<u4v_any *>(p));
    else *reinterpret_cast<u4v_any *>(p) = v;
}

// Eight neighbouring elements, the unit of every vector access here, as they lie in memory: NW words of bf16 pairs (4) or float32 (8)
template <bool BF16>
struct Eight {
    static constexpr int NW = BF16 ? 4 : 8;
    uint32_t w[NW];

    __device__ __forceinline__ float at(int j) const
    {
        if constexpr (BF16) return bits_f((j & 1) ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16);
        else return bits_f(w[j]);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int k = 0; k < NW; ++k) w[k] = 0;
    }
    // values that the compiler must not connect with earlier uses of them
    __device__ __forceinline__ void opaque()
    {
#pragma unroll
        for (int k = 0; k < NW; ++k) asm volatile("" : "+v"(w[k]));
    }
    // the first n of eight elements from p (n >= 8: all, n <= 0: none), the others 0
    template <bool ONCE = false>
    __device__ __forceinline__ void load(const uint8_t *p, int64_t n)
    {
        // (zeros first: written beside the load, they would have to wait for it)
        zero();
        if (n >= 8) {
#pragma unroll
            for (int k = 0; k < NW / 4; ++k) {
                const u4v v = load16<ONCE>(p + 16 * k);
                w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
            }
        } else if (n > 0) {
            // (lanes behind the last element do not take a wave through these)
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < n) {
                    if constexpr (BF16) w[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[j] << (16 * (j & 1));
                    else w[j] = reinterpret_cast<const uint32_t *>(p)[j];
                }
        }
    }
    template <bool ONCE = false>
    __device__ __forceinline__ void store(uint8_t *p, int64_t n) const
    {
        if (n >= 8) {
#pragma unroll
            for (int k = 0; k < NW / 4; ++k) store16<ONCE>(p + 16 * k, u4v{w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]});
            return;
        }
        if (n <= 0) return;
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < n) {
                if constexpr (BF16) reinterpret_cast<uint16_t *>(p)[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
                else reinterpret_cast<uint32_t *>(p)[j] = w[j];
            }
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
#pragma unroll
        for (int k = 0; k < NW; ++k) w[k] = BF16 ? pack_bf16(v[2 * k & 7], v[(2 * k + 1) & 7]) : f_bits(v[k & 7]);
    }
};

// Eight elements of a type that is the same for all lanes, from element i of an array
__device__ __forceinline__ void load_eight(float (&v)[8], const void *base, int bf16, int64_t i, int64_t n)
{
    const uint8_t *p = reinterpret_cast<const uint8_t *>(base);
    if (bf16) {
        Eight<true> e;
        e.load(p + 2 * i, n);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = e.at(j);
    } else {
        Eight<false> e;
        e.load(p + 4 * i, n);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = e.at(j);
    }
}
template <bool ONCE = false>
__device__ __forceinline__ void store_eight(const float (&v)[8], void *base, int bf16, int64_t i, int64_t n)
{
    uint8_t *p = reinterpret_cast<uint8_t *>(base);
    if (bf16) {
        Eight<true> e;
        e.set(v);
        e.template store<ONCE>(p + 2 * i, n);
    } else {
        Eight<false> e;
        e.set(v);
        e.store(p + 4 * i, n);
    }
}

// Sum over the LANES lanes that hold one row (a power of two), the same value in each; the order
// of the additions is fixed.
template <int LANES = 64>
__device__ __forceinline__ double lane_sum(double v)
{
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
// Sum over a workgroup; `lds` holds one double a wave and is not in use any more once every wave
// has passed the next barrier.
__device__ __forceinline__ double group_sum(double v, int waves, double *lds)
{
    v = lane_sum(v);
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    for (int i = 0; i < waves; ++i) s += lds[i];
    return s;
}

// Index of a workgroup in a grid that row_grid made (some at its end have none of the work)
constexpr int64_t kGridX = int64_t(1) << 20;
__device__ __forceinline__ int64_t group_index() { return blockIdx.x + blockIdx.y * kGridX; }
inline dim3 row_grid(int64_t groups)
{
    return groups <= kGridX ? dim3((unsigned)groups) : dim3((unsigned)kGridX, (unsigned)((groups + kGridX - 1) / kGridX));
}

// 1 / sqrt(mean + eps), rounded to float32 once
__device__ __forceinline__ float rstd_of(double sum, int64_t cols, double eps)
{
    return (float)(1.0 / __builtin_sqrt(sum / (double)cols + eps));
}

}  // namespace q2d
