// Device helpers of the attention kernels: operand fragments on the matrix cores, LDS
// tiles, and the masks.
//
// Every product runs as D[m][n] += A[m][k] B[k][n] on 32 x 32 output tiles with k in
// steps of 16, and the kernels choose which operand is A so that a softmax row lies in
// one lane pair: lane l holds column n = l % 32 and the 16 rows 8 (i / 4) + 4 (l / 32) +
// i % 4.  A fragment gives lane l row (or column) l % 32 and 8 values of k, which may be
// any 8 as long as A and B agree.  So an output tile turned into the B operand of the
// next product needs no exchange between lanes: its registers 8 s .. 8 s + 7 are k-step
// s, for an A fragment that holds the same rows (column_frag).
//
// float32 operands take eight v_mfma_f32_32x32x2_f32 a step on the same fragments.
#pragma once

#include <math.h>
#include "attention.hpp"
#include "gemm_common.hpp"

namespace q2d {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v8f __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <typename T> struct FragOf;
template <> struct FragOf<__bf16> { typedef bf16x8 type; };
template <> struct FragOf<float> { typedef v8f type; };
template <typename T> using Frag = typename FragOf<T>::type;

__device__ __forceinline__ v16f mma(bf16x8 a, bf16x8 b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ v16f mma(v8f a, v8f b, v16f c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

// registers 8 s .. 8 s + 7 of an output tile as an operand fragment (bf16: to nearest even)
template <typename T>
__device__ __forceinline__ Frag<T> to_frag(const v16f &x, int s)
{
    Frag<T> f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = x[8 * s + j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const v2f v = {x[8 * s + j], x[8 * s + j + 1]};
            const bf16x2v w = __builtin_convertvector(v, bf16x2v);
            f[j] = w[0];
            f[j + 1] = w[1];
        }
    }
    return f;
}

// An LDS tile of rows of DT elements of T, in 16-byte chunks whose place in a row is
// XORed with a function of the row number: neighbouring rows then start on different
// banks, for reads along rows (row_frag: 16 bytes each of up to 32 rows) and across
// them (column_frag: 32 or 64 bytes of 4 neighbouring rows).
template <typename T, int DT>
struct Tile {
    static constexpr int kPer = 16 / sizeof(T);            // elements a chunk
    static constexpr int kChunks = DT / kPer;              // chunks a row
    static constexpr int kRowBytes = DT * sizeof(T);

    static __device__ __forceinline__ int swizzle(int r)
    {
        if constexpr (sizeof(T) == 4) return r & (kChunks == 32 ? 7 : 15);
        else if constexpr (kChunks == 16) return ((r & 3) << 2) | ((r >> 2) & 3);
        else return ((r & 2) << 1) | ((r >> 2) & 3);
    }
    static __device__ __forceinline__ int offset(int r, int chunk) { return r * kRowBytes + ((chunk ^ swizzle(r)) << 4); }

    // 8 elements 16 ks + 8 h .. of row r (h = lane / 32)
    static __device__ __forceinline__ Frag<T> row_frag(const uint8_t *t, int r, int ks, int h)
    {
        if constexpr (sizeof(T) == 2) {
            return *reinterpret_cast<const bf16x8 *>(t + offset(r, 2 * ks + h));
        } else {
            const v4f a = *reinterpret_cast<const v4f *>(t + offset(r, 4 * ks + 2 * h));
            const v4f b = *reinterpret_cast<const v4f *>(t + offset(r, 4 * ks + 2 * h + 1));
            return v8f{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        }
    }

    // column 32 dt + lane % 32, rows r0 + 4 h + 0..3 and r0 + 8 + 4 h + 0..3
    static __device__ __forceinline__ Frag<T> column_frag(const uint8_t *t, int r0, int dt, int lane)
    {
        const int h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            // ds_read_b64_tr_b16 hands lane i of each 16 the i-th column of a 4 x 16 block
            // whose rows the lanes 4 r .. 4 r + 3 point at
            const int i = lane & 15, r = r0 + 4 * h + (i >> 2);
            const int chunk = 4 * dt + 2 * ((lane >> 4) & 1) + ((i >> 1) & 1), half = (i & 1) << 3;
            typedef __attribute__((address_space(3))) v4s *lp;
            const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t *)t;
            const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(uintptr_t)(base + offset(r, chunk) + half));
            const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(uintptr_t)(base + offset(r + 8, chunk) + half));
            const bf16x4 x = __builtin_bit_cast(bf16x4, a), y = __builtin_bit_cast(bf16x4, b);
            return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            const int d = 32 * dt + (lane & 31);
            v8f f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = r0 + 4 * h + (j & 3) + 2 * (j & 4);
                f[j] = *reinterpret_cast<const float *>(t + offset(r, d >> 2) + ((d & 3) << 2));
            }
            return f;
        }
    }

    static __device__ __forceinline__ float element(const uint8_t *t, int r, int d)
    {
        const uint8_t *p = t + offset(r, d / kPer) + (d % kPer) * sizeof(T);
        if constexpr (sizeof(T) == 4) return *reinterpret_cast<const float *>(p);
        else return bf16_to_f(*reinterpret_cast<const uint16_t *>(p));
    }

    // Fills ROWS rows from row r0 of a matrix of n rows (base; stride in elements, below
    // 2^24) and D columns with NT threads, asynchronously (wait_vmcnt).  Rows from n on
    // repeat row n - 1; columns from D on keep what the tile holds (clear).
    template <int ROWS, int NT>
    static __device__ __forceinline__ void load(uint8_t *t, const T *base, int64_t stride, int r0, int n, int D)
    {
        constexpr int RP = NT / kChunks;                       // rows a pass; swizzle(r + RP) == swizzle(r)
        static_assert(ROWS % RP == 0 && (RP % 16 == 0 || (RP % 8 == 0 && kChunks == 32)), "whole passes");
        const int tid = threadIdx.x, r = tid / kChunks;
        const int d = ((tid % kChunks) ^ swizzle(r)) * kPer;
        const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t *)t +
                             __builtin_amdgcn_readfirstlane(tid & ~63) * 16;
        const uint32_t pitch = (uint32_t)stride * sizeof(T);
        const uint8_t *src = reinterpret_cast<const uint8_t *>(base + (int64_t)r0 * stride);
        if (d >= D) return;
        if (r0 + ROWS <= n) {
            const uint32_t off = r * pitch + d * sizeof(T);
#pragma unroll
            for (int i = 0; i < ROWS / RP; ++i)
                lds_dma16(src + (uint64_t)(i * RP) * pitch, off, lds + i * NT * 16);
        } else {
#pragma unroll
            for (int i = 0; i < ROWS / RP; ++i)
                lds_dma16(src, (uint32_t)min(r + i * RP, n - 1 - r0) * pitch + d * sizeof(T), lds + i * NT * 16);
        }
    }

    // zeros in `bytes` bytes of tiles, for the columns from D on
    template <int NT>
    static __device__ __forceinline__ void clear(uint8_t *t, int bytes)
    {
        for (int i = threadIdx.x * 16; i < bytes; i += NT * 16) *reinterpret_cast<u4v *>(t + i) = u4v{0, 0, 0, 0};
    }

    // whether rows 0 .. ROWS - 1 hold an infinity or a NaN (one wave, the same answer in all lanes)
    template <int ROWS>
    static __device__ __forceinline__ bool non_finite(const uint8_t *t)
    {
        bool bad = false;
#pragma unroll 4
        for (int i = threadIdx.x & 63; i < ROWS * kChunks; i += 64) {
            const u4v v = *reinterpret_cast<const u4v *>(t + i * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 4) bad |= (v[j] & 0x7f800000u) == 0x7f800000u;
                else bad |= (v[j] & 0x7f80u) == 0x7f80u || (v[j] & 0x7f800000u) == 0x7f800000u;
            }
        }
        return __ballot(bad) != 0;
    }
};

// row of an output tile that register i of lane half h holds
__device__ __forceinline__ int tile_row(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// One 8-element operand fragment of a matrix row straight from memory: elements
// 16 ks + 8 h ..; zeros where the row or the columns lie outside
template <typename T>
__device__ __forceinline__ Frag<T> global_frag(const T *row, bool valid, int ks, int h, int D)
{
    const int d = 16 * ks + 8 * h;
    Frag<T> f = {};
    if (valid && d < D) {
        if constexpr (sizeof(T) == 2) {
            f = *reinterpret_cast<const bf16x8 *>(row + d);
        } else {
            const v4f a = *reinterpret_cast<const v4f *>(row + d), b = *reinterpret_cast<const v4f *>(row + d + 4);
            f = v8f{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        }
    }
    return f;
}

// acc (rows d, column n) += sum over the 32 rows r of x's tile that column n sees of
// w[r] X[r0 + r][d], one value at a time: what a matrix product of zeroed weights would
// spoil where a row that is not seen holds an infinity or a NaN.  seen: bit r of a
// column's rows (the same in both lanes of the column).
template <typename T, int DT>
__device__ __forceinline__ void add_rows(v16f *acc, const v16f &w, uint32_t seen, const uint8_t *t, int r0)
{
    const int lane = threadIdx.x & 63, h = lane >> 5;
#pragma unroll 1
    for (int r = 0; r < 32; ++r) {
        // register and half that hold row r
        const int i = 4 * (r >> 3) + (r & 3), from = ((r >> 2) & 1) * 32 + (lane & 31);
        float mine = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) mine = i == j ? w[j] : mine;
        const float wr = __shfl(mine, from);
        if (!((seen >> r) & 1)) continue;
#pragma unroll
        for (int dt = 0; dt < DT / 32; ++dt)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                acc[dt][j] += wr * Tile<T, DT>::element(t, r0 + r, 32 * dt + tile_row(j, h));
                asm volatile("" ::: "memory");          // one read at a time: registers, not speed
            }
    }
}

// ---------------------------------------------------------------- masks

// What the masks leave between query positions [p0, p1] and keys [j0, j1]: nothing, some
// or all pairs.  (qmin, qmax), (kmin, kmax): ranges of their document numbers.
struct Seen { bool any, all; };

__device__ __forceinline__ Seen classify(const AttentionMask &m, int prefix, int p0, int p1, int j0, int j1,
                                         int qmin, int qmax, int kmin, int kmax)
{
    bool any = true, all = true;
    if (m.causal) {
        any = j0 <= p1;
        all = j1 <= p0;
    }
    if (m.window) {
        any = any && p0 - j1 < m.window;
        all = all && p1 - j0 < m.window;
        if (!m.causal) {
            any = any && j0 - p1 < m.window;
            all = all && j1 - p0 < m.window;
        }
    }
    any = any || j0 < prefix;
    all = all || j1 < prefix;
    if (m.documents) {
        any = any && qmin <= kmax && kmin <= qmax && kmax >= 0 && qmax >= 0;
        all = all && qmin == qmax && kmin == kmax && qmin == kmin && qmin >= 0;
    }
    return {any, all && any};
}

// Tiles of one loop axis that a workgroup visits, 64 at a time: lane t classifies tile
// base + t, and three ballots hold what the workgroup and this wave see of them.
struct Schedule {
    uint64_t visit = 0, any = 0, all = 0;
    int base = -64, cur = -1;
    bool wave_any = false, wave_all = false;

    // next visited tile below `end`, or -1 (the same in all waves); f(tile) -> {of the
    // workgroup, of this wave}
    template <typename F>
    __device__ __forceinline__ int next(int end, F &&f)
    {
        while (!visit) {
            base += 64;
            if (base >= end) return -1;
            const int t = base + (threadIdx.x & 63);
            Seen g = {false, false}, w = {false, false};
            if (t < end) f(t, g, w);
            visit = __ballot(g.any);
            any = __ballot(w.any);
            all = __ballot(w.all);
        }
        const int b = __builtin_ctzll(visit);
        visit &= visit - 1;
        wave_any = (any >> b) & 1;
        wave_all = (all >> b) & 1;
        return base + b;
    }
};

// Interval of the other side's positions that one side's position sees, apart from the prefix
__device__ __forceinline__ void seen_by_query(const AttentionMask &m, int p, int &lo, int &hi)
{
    lo = m.window ? p - m.window + 1 : INT32_MIN;
    hi = m.causal ? p + 1 : (m.window ? p + m.window : INT32_MAX);
}
__device__ __forceinline__ void seen_by_key(const AttentionMask &m, int prefix, int j, int &lo, int &hi)
{
    lo = m.causal ? j : (m.window ? j - m.window + 1 : INT32_MIN);
    hi = m.window ? j + m.window : INT32_MAX;
    if (j < prefix) { lo = INT32_MIN; hi = INT32_MAX; }
}

// Document range of the positions [p0, p1] from the ranges of 64 positions; positions
// below zero have no document
__device__ __forceinline__ int2 range_of(const int2 *ranges, int p0, int p1)
{
    if (p1 < 0) return make_int2(-1, -1);
    int2 r = ranges[(p0 < 0 ? 0 : p0) >> 6];
    for (int i = ((p0 < 0 ? 0 : p0) >> 6) + 1; i <= p1 >> 6; ++i) {
        const int2 s = ranges[i];
        r.x = min(r.x, s.x);
        r.y = max(r.y, s.y);
    }
    if (p0 < 0) r.x = min(r.x, -1);
    return r;
}

// Scores are kept as z, in units whose exponent of two is c z: z = s / (scale) and c =
// scale log2 e, or with a cap z = tanh and c = cap log2 e; a distance bias enters z as
// slope log2 e / c.
struct ScoreMap {
    float c, k1, slope;
};
__device__ __forceinline__ ScoreMap score_map(const AttentionMask &m, int hq)
{
    ScoreMap s;
    s.c = (m.cap > 0.f ? m.cap : m.scale) * kLog2e;
    s.k1 = m.cap > 0.f ? m.scale / m.cap : 1.f;
    s.slope = m.slopes ? m.slopes[hq] * kLog2e / s.c : 0.f;
    return s;
}

__device__ __forceinline__ float tanh_of(float x, bool precise)
{
    if (precise) return tanhf(x);
    // 1 - 2 / (e^2x + 1): off by about 2^-23 of 1, far below the bf16 operands' rounding
    return 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * (2.f * kLog2e)));
}

// 4 neighbouring elements to memory, rounded to nearest even for bf16
__device__ __forceinline__ void store4(float *p, float x0, float x1, float x2, float x3)
{
    *reinterpret_cast<v4f *>(p) = v4f{x0, x1, x2, x3};
}
__device__ __forceinline__ void store4(__bf16 *p, float x0, float x1, float x2, float x3)
{
    *reinterpret_cast<bf16x4 *>(p) = __builtin_convertvector(v4f{x0, x1, x2, x3}, bf16x4);
}

// a column of output tiles [d][column] times f into a row of memory
template <typename T, int DS>
__device__ __forceinline__ void store_columns(T *out, const v16f *x, float f, int h, int D)
{
#pragma unroll
    for (int dt = 0; dt < DS; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * dt + 8 * g + 4 * h;
            if (d < D) store4(out + d, x[dt][4 * g] * f, x[dt][4 * g + 1] * f, x[dt][4 * g + 2] * f, x[dt][4 * g + 3] * f);
        }
}

// Workgroup -> (head of batch, tile): each XCD takes a contiguous range of the heads, so
// that the keys and values of a head are read into one L2
__device__ __forceinline__ void head_tile(uint32_t bid, uint32_t n, uint32_t tiles, uint32_t &head, uint32_t &tile)
{
    const uint32_t xcd = bid % kXcds, local = bid / kXcds, per = n / kXcds, rem = n % kXcds;
    const uint32_t t = xcd * per + (xcd < rem ? xcd : rem) + local;
    head = t / tiles;
    tile = t % tiles;
}

}  // namespace
}  // namespace q2d
