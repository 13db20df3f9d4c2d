// Quantized operands of a root-mean-square norm, from the rows and their statistics.
//
// The work split is the quantizers': a workgroup of eight waves owns a 128 x 256 tile, a wave a
// 32 x 128 strip of it, a lane an 8 x 8 sub-block (rows 8 * (lane / 16) .. + 7, columns 8 * (lane %
// 16) .. + 7).  The lane forms y = (h * rstd) * w in float32 and converts it to each format that
// is wanted, so h is read once for all of them.  A 1 x 32 block spans the 4 lanes that differ in
// lane bits 0-1, a 32 x 1 block those that differ in bits 4-5, a 32 x 32 block all 16.
//
// 16384 x 4096 bfloat16 in FP4 and MXFP8, both orientations: 62 us (134 MB read, 205 written, 5.5
// TB/s; 128 registers hold four waves a SIMD, of 156 it took 88 us).  Strips of a few rows take 4-5 us,
// which is a lone wave's 1300 to 2500 instructions.
#include "norm_common.hpp"
#include "norms.hpp"

namespace q2d {

namespace {

// byte of a block's scale: its exponent, or 0xFF for a block that is not finite
__device__ __forceinline__ uint8_t scale_byte(uint32_t amax, int e) { return amax < 0x7F800000u ? (uint8_t)(e + 127) : (uint8_t)0xFF; }
__device__ __forceinline__ float pow2(int e) { return bits_f((uint32_t)(127 + e) << 23); }

// maximum over the 4 lanes of a 1 x 32 block (bits 0-1 of the lane), and of a 32 x 1 block (bits 4-5)
__device__ __forceinline__ uint32_t row_max(uint32_t m)
{
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp((int)m, (int)m, 0xB1, 0xF, 0xF, false));     // quad_perm 1 0 3 2
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp((int)m, (int)m, 0x4E, 0xF, 0xF, false));  // quad_perm 2 3 0 1
}
__device__ __forceinline__ uint32_t column_max(uint32_t m)
{
    // (the swaps leave the pair's two values in the same lane)
    const auto a = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return max((uint32_t)b[0], (uint32_t)b[1]);
}

// 16 bytes of codes from four words of a staged line (their pitch is odd: no 16-byte read)
template <bool ONCE>
__device__ __forceinline__ void store_codes(uint8_t *p, const uint32_t *words)
{
    const u4v v = {words[0], words[1], words[2], words[3]};
    if constexpr (ONCE) __builtin_nontemporal_store(v, reinterpret_cast<u4v *>(p));
    else *reinterpret_cast<u4v *>(p) = v;
}

__device__ __forceinline__ uint32_t fp4_word(const uint32_t (&v)[8], float scale)
{
    uint32_t w = 0;
    w = rtn_pair_f32<0>(w, v[0], v[1], scale);
    w = rtn_pair_f32<1>(w, v[2], v[3], scale);
    w = rtn_pair_f32<2>(w, v[4], v[5], scale);
    return rtn_pair_f32<3>(w, v[6], v[7], scale);
}
__device__ __forceinline__ uint2 fp8_words(const uint32_t (&v)[8], float scale)
{
    uint32_t lo = 0, hi = 0;
    lo = fp8_pair_f32<false>(lo, v[0], v[1], scale);
    lo = fp8_pair_f32<true>(lo, v[2], v[3], scale);
    hi = fp8_pair_f32<false>(hi, v[4], v[5], scale);
    hi = fp8_pair_f32<true>(hi, v[6], v[7], scale);
    return make_uint2(lo, hi);
}

// y = (h * rstd) * w of a sub-block, 0 outside the matrix (rows, cols: what it has from here on):
// a weight or a row that is not finite must not reach past it
template <bool HB>
__device__ __forceinline__ void norm_sub_block(uint32_t (&y)[8][8], const Eight<HB> (&h)[8], const float (&w)[8], const float (&rstd)[8],
                                               int64_t rows, int64_t cols)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) y[i][j] = f_bits((h[i].at(j) * rstd[i]) * w[j]);
    if (__builtin_amdgcn_ballot_w64(rows < 8 || cols < 8) != 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) y[i][j] = i < rows && j < cols ? y[i][j] : 0u;
    }
}

// A workgroup's part of an operand: WR x WC strips, one a wave, from y of each lane's sub-block (0
// outside the matrix) at (r0, c0); tr and tc count tiles of this size.
template <int FP4, bool MX, int WR, int WC, bool ONCE>
__device__ __forceinline__ void store_operands(const NormQuantArgs &a, const uint32_t (&y)[8][8], const int64_t tr, const int64_t tc)
{
    constexpr int kRows = 32 * WR, kCols = 128 * WC, kThreads = 64 * WR * WC;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wr = wave / WC, wc = wave % WC, rg = lane >> 4, cc = lane & 15;
    const int64_t r0 = tr * kRows + wr * 32 + 8 * rg, c0 = tc * kCols + wc * 128 + 8 * cc;

    // ---- convert (block maxima on |bits|: NaN > inf > finite, as unsigned integers), one format
    // and direction after the other, so that little lives beside y
    constexpr bool BLOCKS = FP4 == 1, LINES = FP4 == 2;
    __shared__ uint32_t st4_r[FP4 ? kRows : 1][16 * WC + 1];
    __shared__ uint32_t st4_c[FP4 ? kCols : 1][4 * WR + 1];
    __shared__ uint8_t st4_rs[LINES ? kRows : 1][4 * WC], st4_cs[LINES ? kCols : 1][WR];
    __shared__ uint32_t st8_c[MX ? kCols : 1][8 * WR + 1];
    __shared__ uint8_t st8_rs[MX ? kRows : 1][4 * WC], st8_cs[MX ? kCols : 1][WR];
    const int rl = wr * 32 + 8 * rg, cl = wc * 128 + 8 * cc;
    uint32_t am = 0;
    if constexpr (BLOCKS) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) am = max(am, y[i][j] & 0x7FFFFFFFu);
        am = column_max(row_max(am));
        if (WR == 4 && a.block == 64) {
            // the block beside it in this wave, then the paired wave's strip
            __shared__ uint32_t am64[4][4];
            am = max(am, (uint32_t)__shfl_xor((int)am, 4));
            if (rg == 0 && (cc & 7) == 0) am64[wr][wc * 2 + (cc >> 3)] = am;
            __syncthreads();
            am = max(am, am64[wr ^ 1][wc * 2 + (cc >> 3)]);
        }
        const float scale = pow2(fp4_block_exponent(am));
        uint32_t rowp[8], colp[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) rowp[i] = am < 0x7F800000u ? fp4_word(y[i], scale) : 0u;
        nibble_transpose8(rowp, colp);
#pragma unroll
        for (int i = 0; i < 8; ++i) st4_r[rl + i][wc * 16 + cc] = rowp[i];
#pragma unroll
        for (int j = 0; j < 8; ++j) st4_c[cl + j][wr * 4 + rg] = colp[j];
    }
    if constexpr (LINES || MX) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, y[i][j] & 0x7FFFFFFFu);
            m = row_max(m);
            const bool finite = m < 0x7F800000u;
            if constexpr (LINES) {
                const int e = fp4_block_exponent(m);
                st4_r[rl + i][wc * 16 + cc] = finite ? fp4_word(y[i], pow2(e)) : 0u;
                if ((cc & 3) == 0) st4_rs[rl + i][wc * 4 + (cc >> 2)] = scale_byte(m, e);
            }
            if constexpr (MX) {
                const int e = fp8_block_exponent(m);
                const uint2 w = finite ? fp8_words(y[i], pow2(e)) : make_uint2(0, 0);
                if (a.q8.codes && r0 + i < a.rows && c0 < a.cols_pad) *reinterpret_cast<uint2 *>(a.q8.codes + (r0 + i) * a.q8.ld_codes + c0) = w;
                if ((cc & 3) == 0) st8_rs[rl + i][wc * 4 + (cc >> 2)] = scale_byte(m, e);
            }
        }
        // (serving wants the rowwise copies alone: 64 x 4096 in FP4 and MXFP8
        // with the rows kernel 8.2 us, so 7.4)
        const bool columns = (LINES && a.q4.codes_t) || (MX && a.q8.codes_t);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (!columns) break;
            const uint32_t col[8] = {y[0][j], y[1][j], y[2][j], y[3][j], y[4][j], y[5][j], y[6][j], y[7][j]};
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, col[i] & 0x7FFFFFFFu);
            m = column_max(m);
            const bool finite = m < 0x7F800000u;
            if constexpr (LINES) {
                const int e = fp4_block_exponent(m);
                st4_c[cl + j][wr * 4 + rg] = finite ? fp4_word(col, pow2(e)) : 0u;
                if (rg == 0) st4_cs[cl + j][wr] = scale_byte(m, e);
            }
            if constexpr (MX) {
                const int e = fp8_block_exponent(m);
                const uint2 w = finite ? fp8_words(col, pow2(e)) : make_uint2(0, 0);
                st8_c[cl + j][wr * 8 + 2 * rg] = w.x;
                st8_c[cl + j][wr * 8 + 2 * rg + 1] = w.y;
                if (rg == 0) st8_cs[cl + j][wr] = scale_byte(m, e);
            }
        }
    }
    __syncthreads();

    // ---- stores, 16 bytes a lane
    if constexpr (FP4 != 0) {
        const QuantOut &q = a.q4;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int item = threadIdx.x + kThreads * p;
            if (q.codes) {
                const int line = item / (4 * WC), part = item % (4 * WC);
                const int64_t r = tr * kRows + line;
                if (r < a.rows && tc * kCols + part * 32 < a.cols_pad)
                    store_codes<false>(q.codes + r * q.ld_codes + tc * (kCols / 2) + part * 16, &st4_r[line][4 * part]);
            }
            if (q.codes_t) {
                const int line = item / WR, part = item % WR;
                const int64_t c = tc * kCols + line;
                if (c < a.cols) store_codes<ONCE>(q.codes_t + c * q.ld_codes_t + tr * (kRows / 2) + part * 16, &st4_c[line][4 * part]);
            }
        }
    }
    if constexpr (BLOCKS) {
        if (rg == 0 && (cc & 3) == 0 && tc * kCols + wc * 128 < a.cols_pad) {
            const QuantOut &q = a.q4;
            const uint8_t byte = scale_byte(am, fp4_block_exponent(am));
            const int64_t rb = r0 >> 5, cb = c0 >> 5;
            if (q.codes && r0 < a.rows) q.scales[rb * q.ld_scales + cb] = byte;
            if (q.codes_t && c0 < a.cols) q.scales_t[cb * q.ld_scales_t + rb] = byte;
        }
    }
    if constexpr (MX) {
        const QuantOut &q = a.q8;
        if (q.codes_t) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const int item = threadIdx.x + kThreads * p;
                const int line = item / (2 * WR), part = item % (2 * WR);
                const int64_t c = tc * kCols + line;
                if (c < a.cols) store_codes<ONCE>(q.codes_t + c * q.ld_codes_t + tr * kRows + part * 16, &st8_c[line][4 * part]);
            }
        }
    }
    // scale words of rows and columns (1D FP4: K-tile major); of a strip of its own one byte a column
    if constexpr (LINES || MX) {
        for (int t = threadIdx.x; t < kRows; t += kThreads) {
            const int64_t r = tr * kRows + t;
            if (r >= a.rows) continue;
#pragma unroll
            for (int k = 0; k < WC; ++k) {
                const int64_t word = tc * WC + k;
                if (word * 128 >= a.cols_pad) continue;
                if constexpr (LINES) {
                    if (a.q4.codes) *reinterpret_cast<uint32_t *>(a.q4.scales + word * a.q4.ld_scales + 4 * r) = *reinterpret_cast<const uint32_t *>(&st4_rs[t][4 * k]);
                }
                if constexpr (MX) {
                    if (a.q8.codes) *reinterpret_cast<uint32_t *>(a.q8.scales + r * a.q8.ld_scales + 4 * word) = *reinterpret_cast<const uint32_t *>(&st8_rs[t][4 * k]);
                }
            }
        }
        for (int t = kThreads - 1 - threadIdx.x; t < kCols; t += kThreads) {
            const int64_t c = tc * kCols + t;
            if (c >= a.cols) continue;
            if constexpr (LINES) {
                const QuantOut &q = a.q4;
                if (q.codes_t) {
                    if constexpr (WR == 4) *reinterpret_cast<uint32_t *>(q.scales_t + tr * q.ld_scales_t + 4 * c) = *reinterpret_cast<const uint32_t *>(&st4_cs[t][0]);
                    else q.scales_t[(tr >> 2) * q.ld_scales_t + 4 * c + (tr & 3)] = st4_cs[t][0];
                }
            }
            if constexpr (MX) {
                const QuantOut &q = a.q8;
                if (q.codes_t) {
                    if constexpr (WR == 4) *reinterpret_cast<uint32_t *>(q.scales_t + c * q.ld_scales_t + tr * 4) = *reinterpret_cast<const uint32_t *>(&st8_cs[t][0]);
                    else q.scales_t[c * q.ld_scales_t + tr] = st8_cs[t][0];
                }
            }
        }
    }
}

// Both formats by one workgroup, or, in strips, by one each (gridDim.y 2): a lone wave takes 4
// cycles an instruction, and the conversions are most of its time (64 x 4096 in FP4 and
// MXFP8 with the rows kernel 9.9 us, so 9.4)
template <int FP4, bool MX, int WR, int WC, bool ONCE>
__device__ __forceinline__ void store_formats(const NormQuantArgs &a, const uint32_t (&y)[8][8], const int64_t tr, const int64_t tc)
{
    if constexpr (FP4 != 0 && MX && WR == 1) {
        if (blockIdx.y == 0) store_operands<FP4, false, WR, WC, ONCE>(a, y, tr, tc);
        else store_operands<0, true, WR, WC, ONCE>(a, y, tr, tc);
    } else {
        store_operands<FP4, MX, WR, WC, ONCE>(a, y, tr, tc);
    }
}

// From h and its rows' statistics.  HB: h is bfloat16.  ALIGNED: its rows are on 16-byte boundaries.
// FP4: 0 none, 1 2D blocks, 2 1D blocks.  ONCE: the transposed codes go past the cache.
template <bool HB, bool ALIGNED, int FP4, bool MX, int WR, int WC, bool ONCE>
__global__ __launch_bounds__(64 * WR * WC) __attribute__((amdgpu_waves_per_eu(WR == 4 ? 4 : 1))) void rmsnorm_quantize_kernel(const NormQuantArgs a)
{
    static_assert((WR == 4 && WC == 2) || (WR == 1 && WC == 1), "a tile, or a strip of its own");
    constexpr int E = HB ? 2 : 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tiles_c = (a.cols_pad + 128 * WC - 1) / (128 * WC);
    // (the last rows first: the rows kernel has written them last, and the cache still holds some
    // of them.  16384 x 4096 float32 in FP4 with the rows kernel 189 us, so 178)
    // (strips are in a grid of one dimension: its second is the format)
    const int64_t tile = (a.rows_pad / (32 * WR)) * tiles_c - 1 - (WR == 1 ? (int64_t)blockIdx.x : group_index());
    if (tile < 0) return;
    const int64_t tr = tile / tiles_c, tc = tile - tr * tiles_c;
    const int64_t r0 = tr * (32 * WR) + (wave / WC) * 32 + 8 * (lane >> 4), c0 = tc * (128 * WC) + (wave % WC) * 128 + 8 * (lane & 15);
    const int64_t cols = a.cols - c0;

    uint32_t y[8][8];
    {
        Eight<HB> h[8];
        const uint8_t *p = reinterpret_cast<const uint8_t *>(a.h) + (r0 * a.ldh + c0) * E;
        if constexpr (ALIGNED) {
            uint32_t v[8][2 * E];
            load_sub_block<E, true, 0>(v, p, a.ldh * E, a.rows - r0, cols);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int k = 0; k < 2 * E; ++k) h[i].w[k] = v[i][k];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i].load(p + i * a.ldh * E, r0 + i < a.rows ? cols : 0);
        }
        float w[8], rstd[8];
        load_run(w, a.w, a.w_bf16, c0, cols);
        load_run(rstd, a.rstd, 0, r0, a.rows - r0);
        norm_sub_block(y, h, w, rstd, a.rows - r0, cols);
    }
    store_formats<FP4, MX, WR, WC, ONCE>(a, y, tr, tc);
}

// f(FP4, MX) for the formats of a call
template <typename F>
void for_formats(const NormQuantArgs &a, F f)
{
    switch (a.fp4 * 2 + (a.mx ? 1 : 0)) {
    case 1: f(std::integral_constant<int, 0>{}, std::true_type{}); break;
    case 2: f(std::integral_constant<int, 1>{}, std::false_type{}); break;
    case 3: f(std::integral_constant<int, 1>{}, std::true_type{}); break;
    case 4: f(std::integral_constant<int, 2>{}, std::false_type{}); break;
    default: f(std::integral_constant<int, 2>{}, std::true_type{}); break;
    }
}

template <bool HB, bool ALIGNED, int WR, int WC, bool ONCE>
void launch_w(const NormQuantArgs &a, hipStream_t s)
{
    const int64_t blocks = (a.rows_pad / (32 * WR)) * ((a.cols_pad + 128 * WC - 1) / (128 * WC));
    const dim3 grid = WR == 1 ? dim3((unsigned)blocks, a.fp4 && a.mx ? 2 : 1) : row_grid(blocks);
    for_formats(a, [&](auto fp4, auto mx) {
        hipLaunchKernelGGL((rmsnorm_quantize_kernel<HB, ALIGNED, decltype(fp4)::value, decltype(mx)::value, WR, WC, ONCE>),
                           grid, dim3(64 * WR * WC), 0, s, a);
    });
}

// Up to 128 tiles, a strip a workgroup (64 x 64 blocks reach over two strips and stay in tiles)
template <bool HB, bool ALIGNED>
void launch_v(const NormQuantArgs &a, hipStream_t s)
{
    const bool strips = a.block == 32 && (a.rows_pad / 128) * ((a.cols_pad + 255) / 256) <= 128;
    // Transposed codes of 48 MB or more go past the cache: the backward pass reads them, long after,
    // and the rowwise ones stay for the GEMM that comes next.  16384 x 4096 bfloat16 in FP4 and MXFP8
    // with the rows kernel 131 -> 123 us, with two GEMMs behind it 230 -> 219; 32768 x 4096 in FP4 and
    // a GEMM 263 -> 257; half of that, 33 MB, 132.8 -> 133.2.  (A call that reads the transposed copies
    // at once pays for it: with q2d_dequantize of all four 250 -> 270.)
    const int64_t bytes = a.rows * a.cols * ((a.fp4 && a.q4.codes_t ? 1 : 0) + (a.mx && a.q8.codes_t ? 2 : 0)) / 2;
    if (strips) launch_w<HB, ALIGNED, 1, 1, false>(a, s);
    else if (bytes >= int64_t(48) << 20) launch_w<HB, ALIGNED, 4, 2, true>(a, s);
    else launch_w<HB, ALIGNED, 4, 2, false>(a, s);
}

}  // namespace

hipError_t launch_rmsnorm_quantize(const NormQuantArgs &a, hipStream_t stream)
{
    const bool aligned = reinterpret_cast<uintptr_t>(a.h) % 16 == 0 && a.ldh % (a.h_bf16 ? 8 : 4) == 0;
    if (a.h_bf16) {
        if (aligned) launch_v<true, true>(a, stream);
        else launch_v<true, false>(a, stream);
    } else {
        if (aligned) launch_v<false, true>(a, stream);
        else launch_v<false, false>(a, stream);
    }
    return hipGetLastError();
}

}  // namespace q2d
