// Dequantization of one stored copy of a quantized matrix back to R x C values,
// with the per-element scale exponent alongside (optional).
//
// This is what each GEMM of a linear layer effectively multiplies (Sec. 2,
// "Bias induced by scale inconsistency": the forward copy X_fwd = round(X/S_fwd)
// S_fwd and the backward copy X_bwd = round(X/S_bwd) S_bwd).  Dequantizing both
// copies of one tensor in the same R x C orientation gives the scale-difference
// and effective-deviation maps of the forward/backward comparison (Fig. 1): zero
// for 2D blocks, non-zero for 1D blocks.
//
// The quantizers' work split: a workgroup of eight waves owns a 128 x 256 tile, a wave a 32 x 128
// strip of it, a lane an 8 x 8 sub-block (rows 8 * (lane / 16) .. + 7, columns 8 * (lane % 16) ..
// + 7); few tiles are cut into one-wave workgroups.  A row-packed copy is read straight into
// the lanes.  A transposed copy (stored K = rows) goes through LDS, from where a lane takes its
// eight columns' words and transposes them in registers.  A lane stores eight neighbouring
// elements of a row at a time (16 bytes of bfloat16, at any address).  Values are exact in float32
// (an E2M1 or E4M3 code times a power of two, rounded once only when it leaves float32 range);
// bfloat16 output is the round-to-nearest-even of that value.
//
// Element by element from LDS, with the scales read beside it, the transposed MXFP8 copy of
// 16384 x 4096 took 139 us as bfloat16 and 164 as float32; now 35 and 85 (5.9 and 4.0 TB/s).
#include "device_common.hpp"
#include "kernels.hpp"
#include "norm_common.hpp"

namespace q2d {

namespace {

constexpr uint32_t kNaN = 0x7FC00000u;

// a scale byte as the power of two that it stands for
__device__ __forceinline__ float scale_value(uint32_t byte)
{
    return bits_f(byte == 0xFFu ? kNaN : byte ? byte << 23 : 0x00400000u);
}

// its exponent as int8, -128 for 0xFF: both are the byte less 127
__device__ __forceinline__ uint8_t exponent(uint32_t byte) { return (uint8_t)(byte - 127u); }

// The first n of eight exponents at any address, together where all are wanted.  (One byte at a time,
// 16384 x 4096 float32 with exponents took 113 us, MXFP8 132; so 85 and 100)
__device__ __forceinline__ void store_exponents(int8_t *p, const uint8_t (&b)[8], int64_t n)
{
    typedef u2v any __attribute__((aligned(1)));
    if (n >= 8) {
        u2v v;
#pragma unroll
        for (int k = 0; k < 2; ++k) v[k] = b[4 * k] | b[4 * k + 1] << 8 | b[4 * k + 2] << 16 | (uint32_t)b[4 * k + 3] << 24;
        *reinterpret_cast<any *>(p) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < n) p[j] = (int8_t)b[j];
    }
}

// values of eight E2M1 nibbles, times 1
__device__ __forceinline__ void fp4_values(uint32_t w, float (&v)[8])
{
    const f32v2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1);
    const f32v2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y; v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
}

// values of four E4M3FN bytes (S.1111.111 is a NaN of either sign)
__device__ __forceinline__ void fp8_values(uint32_t w, float *v)
{
    const f32v2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}

// whether a wave has a NaN code: seven ones and one more carry into a byte's highest bit
template <int WORDS>
__device__ __forceinline__ bool fp8_nan(const uint32_t (&w)[8][WORDS])
{
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int k = 0; k < WORDS; ++k) any |= (w[i][k] & 0x7F7F7F7Fu) + 0x01010101u;
    return __builtin_amdgcn_ballot_w64((any & 0x80808080u) != 0) != 0;
}

// 4 x 4 transpose of bytes: byte j of in[i] becomes byte i of out[j]
__device__ __forceinline__ void byte_transpose4(const uint32_t (&in)[4], uint32_t (&out)[4])
{
    const uint32_t a = __builtin_amdgcn_perm(in[1], in[0], 0x05010400u), b = __builtin_amdgcn_perm(in[3], in[2], 0x05010400u);
    const uint32_t c = __builtin_amdgcn_perm(in[1], in[0], 0x07030602u), d = __builtin_amdgcn_perm(in[3], in[2], 0x07030602u);
    out[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(d, c, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

// FMT: 0 = FP4 2D blocks, 1 = MXFP8, 2 = FP4 1D blocks.  TRANS: the copy is stored with K = rows
// (element (r, c) in stored row c).  WR x WC strips, one a wave.  ONCE: the output is more than the
// cache holds.
template <int FMT, bool TRANS, bool BF16, int WR, int WC, bool ONCE = false>
__global__ __launch_bounds__(64 * WR * WC) void dequantize_kernel(const DequantArgs a)
{
    constexpr int kRows = 32 * WR, kCols = 128 * WC, kThreads = 64 * WR * WC;
    constexpr int kWords = FMT == 1 ? 2 : 1;             // words of eight codes
    const int64_t tiles_c = (a.cols + kCols - 1) / kCols;
    const int64_t tile = group_index(), tr = tile / tiles_c, tc = tile - tr * tiles_c;
    if (tr * kRows >= a.rows) return;                    // (a grid of two dimensions may hold more)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wr = wave / WC, wc = wave % WC, rg = lane >> 4, cc = lane & 15;
    const int64_t r0 = tr * kRows + wr * 32 + 8 * rg, c0 = tc * kCols + wc * 128 + 8 * cc;
    const bool some = r0 < a.rows && c0 < a.cols;

    // ---- the scale bytes of the sub-block's rows (row-packed copy) or columns, one for a 2D block.
    // A tile's columns in 1D blocks have theirs side by side, a word for four blocks, and these go
    // through LDS (8192 x 2048 11.8 us, so 9.5; MXFP8's words lie apart and gained nothing)
    constexpr int kScales = FMT == 0 ? 1 : 8;
    constexpr bool STAGED = FMT == 2 && TRANS && WR == 4;
    __shared__ uint32_t words[STAGED ? kCols : 1];
    uint32_t sb[kScales];
    if constexpr (STAGED) {
        const int64_t s = tc * kCols + threadIdx.x;
        if (threadIdx.x < kCols) words[threadIdx.x] = s < a.cols ? *reinterpret_cast<const uint32_t *>(a.scales + tr * a.ld_scales + 4 * s) : 0u;
    } else {
#pragma unroll
        for (int i = 0; i < kScales; ++i) {
            const int64_t s = (TRANS ? c0 : r0) + i, k = TRANS ? r0 : c0;
            sb[i] = 0;
            if (!some || (kScales > 1 && s >= (TRANS ? a.cols : a.rows))) continue;
            sb[i] = FMT == 0 ? a.scales[(s >> 5) * a.ld_scales + (k >> 5)]
                  : FMT == 2 ? a.scales[(k >> 7) * a.ld_scales + 4 * s + ((k >> 5) & 3)]
                             : a.scales[s * a.ld_scales + (k >> 5)];
        }
    }

    // ---- the codes: w[i] has the eight of row i
    uint32_t w[8][kWords];
    if constexpr (!TRANS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int k = 0; k < kWords; ++k) w[i][k] = 0;
            if (!some || r0 + i >= a.rows) continue;
            const uint8_t *p = a.codes + (r0 + i) * a.ld_codes + (FMT == 1 ? c0 : c0 / 2);
            if constexpr (FMT == 1) {
                const uint2 q = *reinterpret_cast<const uint2 *>(p);
                w[i][0] = q.x; w[i][kWords - 1] = q.y;
            } else {
                w[i][0] = *reinterpret_cast<const uint32_t *>(p);
            }
        }
    } else {
        // stored rows of kRows codes, 16 bytes a lane
        constexpr int kLine = WR * 4 * kWords, kParts = kLine / 4;         // words, 16-byte parts
        __shared__ uint32_t st[kCols][kLine + 1];
#pragma unroll
        for (int q = 0; q < kCols * kParts / kThreads; ++q) {
            const int item = threadIdx.x + kThreads * q, line = item / kParts, part = item % kParts;
            const int64_t c = tc * kCols + line;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (c < a.cols) v = *reinterpret_cast<const uint4 *>(a.codes + c * a.ld_codes + tr * (4 * kLine) + 16 * part);
            st[line][4 * part] = v.x; st[line][4 * part + 1] = v.y; st[line][4 * part + 2] = v.z; st[line][4 * part + 3] = v.w;
        }
        __syncthreads();
        uint32_t col[8][kWords];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int k = 0; k < kWords; ++k) col[j][k] = st[wc * 128 + 8 * cc + j][(wr * 4 + rg) * kWords + k];
        if constexpr (FMT == 1) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t in[4] = {col[4 * h][k], col[4 * h + 1][k], col[4 * h + 2][k], col[4 * h + 3][k]};
                    uint32_t out[4];
                    byte_transpose4(in, out);
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[4 * k + i][h] = out[i];
                }
        } else {
            uint32_t in[8], out[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) in[j] = col[j][0];
            nibble_transpose8(in, out);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i][0] = out[i];
        }
    }
    if constexpr (STAGED) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sb[i] = (words[wc * 128 + 8 * cc + i] >> (8 * wr)) & 0xFFu;
    }
    // float32 writes are what such a call takes; a workgroup's waves, together to here, write lines that lie
    // together (the transposed copies have a barrier above): 16384 x 11008 FP4 202 us, so 171, MXFP8 227, 189
    if constexpr (!BF16 && !TRANS) __syncthreads();
    if (!some) return;

    float scale[kScales];
#pragma unroll
    for (int i = 0; i < kScales; ++i) scale[i] = scale_value(sb[i]);
    bool nan = false;
    if constexpr (FMT == 1) nan = fp8_nan(w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + i;
        if (r >= a.rows) break;
        float v[8];
        if constexpr (FMT == 1) {
            fp8_values(w[i][0], v);
            fp8_values(w[i][kWords - 1], v + 4);
        } else {
            fp4_values(w[i][0], v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= scale[kScales == 1 ? 0 : TRANS ? j : i];
        if (FMT == 1 && nan) {
            // (the conversion's NaN are negative ones)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = v[j] == v[j] ? v[j] : bits_f(kNaN);
        }
        store_run<ONCE>(v, a.out, BF16, r * a.ldo + c0, a.cols - c0);
        if (a.exps) {
            uint8_t b[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) b[j] = exponent(sb[kScales == 1 ? 0 : TRANS ? j : i]);
            store_exponents(a.exps + r * a.lde + c0, b, a.cols - c0);
        }
    }
}

template <int FMT, bool TRANS, bool BF16>
hipError_t launch_tiles(const DequantArgs &a, hipStream_t s)
{
    auto tiles = [&](int64_t rows, int64_t cols) { return ((a.rows + rows - 1) / rows) * ((a.cols + cols - 1) / cols); };
    // (as the quantizers: up to 128 tiles, a strip a workgroup)
    if (tiles(128, 256) <= 128) {
        hipLaunchKernelGGL((dequantize_kernel<FMT, TRANS, BF16, 1, 1>), dim3((unsigned)tiles(32, 128)), dim3(64), 0, s, a);
    } else {
        // bfloat16 output of 96 MB or more past the cache: 16384 x 4096 FP4 37 -> 26 us, MXFP8 transposed
        // 58 -> 35; with a kernel that reads the output behind it 65 -> 61, half the size 30 -> 34.
        // (float32 stores of eight elements are two to a line and stay)
        const dim3 grid = row_grid(tiles(128, 256)), block(512);
        if constexpr (BF16) {
            if (a.rows * a.cols * 2 >= int64_t(96) << 20) {
                hipLaunchKernelGGL((dequantize_kernel<FMT, TRANS, BF16, 4, 2, true>), grid, block, 0, s, a);
                return hipGetLastError();
            }
        }
        hipLaunchKernelGGL((dequantize_kernel<FMT, TRANS, BF16, 4, 2>), grid, block, 0, s, a);
    }
    return hipGetLastError();
}

template <int FMT, bool TRANS>
hipError_t launch_fmt(const DequantArgs &a, hipStream_t s)
{
    return a.out_bf16 ? launch_tiles<FMT, TRANS, true>(a, s) : launch_tiles<FMT, TRANS, false>(a, s);
}

}  // namespace

hipError_t launch_dequantize(const DequantArgs &a, hipStream_t stream)
{
    switch (a.fmt * 2 + (a.transposed ? 1 : 0)) {
    case 0: return launch_fmt<0, false>(a, stream);
    case 1: return launch_fmt<0, true>(a, stream);
    case 2: return launch_fmt<1, false>(a, stream);
    case 3: return launch_fmt<1, true>(a, stream);
    case 4: return launch_fmt<2, false>(a, stream);
    case 5: return launch_fmt<2, true>(a, stream);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace q2d
