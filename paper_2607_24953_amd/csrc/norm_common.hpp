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

// 8 or 16 bytes (2 or 4 words) at any address of an element: the hardware takes wide accesses there
// too, in the same instructions, so rows need no alignment.  ONCE: of data that is not read or written
// again soon.
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
template <int WORDS> struct Wide;
template <> struct Wide<2> { typedef u2v type; };
template <> struct Wide<4> { typedef u4v type; };
template <int WORDS, bool ONCE>
__device__ __forceinline__ void load_wide(uint32_t *w, const uint8_t *p)
{
    typedef typename Wide<WORDS>::type V;
    typedef V any __attribute__((aligned(2)));
    V v;
    if constexpr (ONCE) v = __builtin_nontemporal_load(reinterpret_cast<const any *>(p));
    else v = *reinterpret_cast<const any *>(p);
#pragma unroll
    for (int k = 0; k < WORDS; ++k) w[k] = v[k];
}
template <int WORDS, bool ONCE>
__device__ __forceinline__ void store_wide(uint8_t *p, const uint32_t *w)
{
    typedef typename Wide<WORDS>::type V;
    typedef V any __attribute__((aligned(2)));
    V v;
#pragma unroll
    for (int k = 0; k < WORDS; ++k) v[k] = w[k];
    if constexpr (ONCE) __builtin_nontemporal_store(v, reinterpret_cast<any *>(p));
    else *reinterpret_cast<any *>(p) = v;
}

// N (4 or 8) neighbouring elements, the unit of every vector access here, as they lie in memory: NW
// words of bf16 pairs or float32
template <bool BF16, int N>
struct Run {
    static constexpr int NW = BF16 ? N / 2 : N, kWide = NW < 4 ? 2 : 4;
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
    // the first n of N elements from p (n >= N: all, n <= 0: none), the others 0
    template <bool ONCE = false>
    __device__ __forceinline__ void load(const uint8_t *p, int64_t n)
    {
        // (zeros first: written beside the load, they would have to wait for it)
        zero();
        if (n >= N) {
#pragma unroll
            for (int k = 0; k < NW; k += kWide) load_wide<kWide, ONCE>(w + k, p + 4 * k);
        } else if (n > 0) {
            // (lanes behind the last element do not take a wave through these)
#pragma unroll
            for (int j = 0; j < N - 1; ++j)
                if (j < n) {
                    if constexpr (BF16) w[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[j] << (16 * (j & 1));
                    else w[j] = reinterpret_cast<const uint32_t *>(p)[j];
                }
        }
    }
    template <bool ONCE = false>
    __device__ __forceinline__ void store(uint8_t *p, int64_t n) const
    {
        if (n >= N) {
#pragma unroll
            for (int k = 0; k < NW; k += kWide) store_wide<kWide, ONCE>(p + 4 * k, w + k);
        } else if (n > 0) {
#pragma unroll
            for (int j = 0; j < N - 1; ++j)
                if (j < n) {
                    if constexpr (BF16) reinterpret_cast<uint16_t *>(p)[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
                    else reinterpret_cast<uint32_t *>(p)[j] = w[j];
                }
        }
    }
    __device__ __forceinline__ void set(const float (&v)[N])
    {
#pragma unroll
        for (int k = 0; k < NW; ++k) w[k] = BF16 ? pack_bf16(v[2 * k % N], v[(2 * k + 1) % N]) : f_bits(v[k % N]);
    }
};
template <bool BF16> using Eight = Run<BF16, 8>;

// N elements of a type that is the same for all lanes, from element i of an array
template <int N>
__device__ __forceinline__ void load_run(float (&v)[N], const void *base, int bf16, int64_t i, int64_t n)
{
    const uint8_t *p = reinterpret_cast<const uint8_t *>(base);
    if (bf16) {
        Run<true, N> e;
        e.load(p + 2 * i, n);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = e.at(j);
    } else {
        Run<false, N> e;
        e.load(p + 4 * i, n);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = e.at(j);
    }
}
template <bool ONCE = false, int N>
__device__ __forceinline__ void store_run(const float (&v)[N], void *base, int bf16, int64_t i, int64_t n)
{
    uint8_t *p = reinterpret_cast<uint8_t *>(base);
    if (bf16) {
        Run<true, N> e;
        e.set(v);
        e.template store<ONCE>(p + 2 * i, n);
    } else {
        Run<false, N> e;
        e.set(v);
        e.template store<ONCE>(p + 4 * i, n);
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
