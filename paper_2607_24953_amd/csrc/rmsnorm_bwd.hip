// Gradient of the root-mean-square norm.
//
// With n = h * rstd and g = dy * w: dx = rstd * (g - n * mean(g n)) + dh, dw = sum over rows of dy n.
// One read of h, dy and dh: a row stays in registers between the sum for its mean and the products
// with it, as in the forward kernel.  A workgroup takes every gridDim.x-th row and keeps its part
// of dw in registers, in 64 bits; the parts lie one behind the other in the workspace and a second
// kernel adds them up.  Every sum has one owner and one order.
//
// The memory bounds it: 16384 x 4096 bfloat16 with dh 86 us (545 MB, 6.3 TB/s) and 5 for the join,
// float32 151 in all; 777 x 2049 8.5 + 3.5.  The statistics of a row and the products with it as two
// kernels, element by element, took 700.  Rows of 8193 to 16384 columns leave one workgroup of up
// to 16 waves to a CU, with nothing to run while it waits at its barrier (2048 x 12288 68 us, 2.9 TB/s).
#include "norm_common.hpp"
#include "norms.hpp"
#include "kernels.hpp"

namespace q2d {

namespace {


// HB, DB: h and dh, dy are bfloat16.  LANES, CH: as in the forward kernel.  ONCE: the rows come from
// memory rather than from the cache.
template <bool HB, bool DB, int LANES, int CH, bool ONCE>
__global__ __launch_bounds__(LANES ? 256 : 1024) void rmsnorm_grad_kernel(const NormGradArgs a, float *part)
{
    constexpr int EH = HB ? 2 : 4, ED = DB ? 2 : 4, N = 16 / EH;
    constexpr int kPer = LANES ? 256 / (LANES ? LANES : 1) : 1;        // rows at a time
    __shared__ double lds[2][16];
    const int t = LANES ? threadIdx.x % (LANES ? LANES : 1) : threadIdx.x, step = LANES ? LANES : blockDim.x;
    const int sub = LANES ? threadIdx.x / (LANES ? LANES : 1) : 0;
    // (two chunks of weights beside two of everything else do not fit 128 registers)
    constexpr bool KEPT = LANES != 0 || CH * N <= 8;
    float w[CH][N];
    double acc[CH][N];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int64_t c = N * (t + k * (int64_t)step);
        if constexpr (KEPT) load_run(w[k], a.w, a.w_bf16, c, a.cols - c);
#pragma unroll
        for (int j = 0; j < N; ++j) acc[k][j] = 0.0;
    }
    int turn = 0;
    for (int64_t first = blockIdx.x * (int64_t)kPer; first < a.rows; first += gridDim.x * (int64_t)kPer, turn ^= 1) {
        const int64_t row = first + sub;
        // (lanes of a row beyond the last one hold nothing)
        const bool some = row < a.rows;
        const int64_t cols = some ? a.cols : 0;
        const uint8_t *hp = reinterpret_cast<const uint8_t *>(a.h) + row * a.ldh * EH;
        const uint8_t *dyp = reinterpret_cast<const uint8_t *>(a.dy) + row * a.lddy * ED;
        const uint8_t *dhp = reinterpret_cast<const uint8_t *>(a.dh) + row * a.lddh * EH;
        uint8_t *dxp = reinterpret_cast<uint8_t *>(a.dx) + row * a.lddx * EH;
        Run<HB, N> h[CH], dh[CH];
        Run<DB, N> dy[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t c = N * (t + k * (int64_t)step);
            h[k].template load<ONCE>(hp + c * EH, cols - c);
            dy[k].template load<ONCE>(dyp + c * ED, cols - c);
            if (a.dh) dh[k].template load<ONCE>(dhp + c * EH, cols - c);
            else dh[k].zero();
        }
        const float rstd = some ? a.rstd[row] : 0.f;
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if constexpr (!KEPT) load_run(w[k], a.w, a.w_bf16, N * (t + k * (int64_t)step), a.cols - N * (t + k * (int64_t)step));
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float n = h[k].at(j) * rstd, d = dy[k].at(j);
                sum = __builtin_fma((double)(d * w[k][j]), (double)n, sum);
                acc[k][j] = __builtin_fma((double)d, (double)n, acc[k][j]);
            }
        }
        if constexpr (LANES) sum = lane_sum<LANES ? LANES : 64>(sum);
        else sum = group_sum(sum, blockDim.x >> 6, lds[turn]);
        const float mean = (float)(sum / (double)a.cols);
        // (n and g are formed again: kept over the sum they would take 32 registers a chunk)
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            h[k].opaque();
            dy[k].opaque();
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t c = N * (t + k * (int64_t)step);
            if (c >= cols) break;
            if constexpr (!KEPT) load_run(w[k], a.w, a.w_bf16, c, a.cols - c);
            float dx[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float n = h[k].at(j) * rstd;
                dx[j] = rstd * (dy[k].at(j) * w[k][j] - n * mean) + dh[k].at(j);
            }
            Run<HB, N> o;
            o.set(dx);
            o.store(dxp + c * EH, cols - c);
        }
    }
    if (!part) return;
    part += blockIdx.x * a.cols;
    if constexpr (LANES) {
        // the rows' lanes of a column, in order
        __shared__ double sums[kPer][N * (LANES ? LANES : 1) + 2];
        for (int k = 0; k < CH; ++k) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < N; ++j) sums[sub][N * t + j] = acc[k][j];
            __syncthreads();
            for (int i = threadIdx.x; i < N * LANES; i += 256) {
                const int64_t c = N * (int64_t)LANES * k + i;
                double s = 0.0;
                for (int p = 0; p < kPer; ++p) s += sums[p][i];
                if (c < a.cols) part[c] = (float)s;
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t c = N * (t + k * (int64_t)step);
            Run<false, N> o;
            float v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = (float)acc[k][j];
            o.set(v);
            o.store(reinterpret_cast<uint8_t *>(part + c), a.cols - c);
        }
    }
}

// Rows that no workgroup's registers hold: their means first
__global__ __launch_bounds__(1024) void rmsnorm_grad_means_kernel(const NormGradArgs a, float *means)
{
    const int64_t row = group_index();
    if (row >= a.rows) return;
    __shared__ double lds[16];
    const float rstd = a.rstd[row];
    double s = 0.0;
    for (int64_t c = 8 * (int64_t)threadIdx.x; c < a.cols; c += 8 * 1024) {
        float d[8], w[8], h[8];
        load_run(d, a.dy, a.dy_bf16, row * a.lddy + c, a.cols - c);
        load_run(w, a.w, a.w_bf16, c, a.cols - c);
        load_run(h, a.h, a.h_bf16, row * a.ldh + c, a.cols - c);
#pragma unroll
        for (int j = 0; j < 8; ++j) s = __builtin_fma((double)(d[j] * w[j]), (double)(h[j] * rstd), s);
    }
    s = group_sum(s, 16, lds);
    if (threadIdx.x == 0) means[row] = (float)(s / (double)a.cols);
}

// .. then 2048 columns of every gridDim.y-th row
__global__ __launch_bounds__(256) void rmsnorm_grad_tile_kernel(const NormGradArgs a, const float *means, float *part)
{
    const int64_t c = 8 * (blockIdx.x * (int64_t)256 + threadIdx.x), n = a.cols - c;
    if (n <= 0) return;
    float w[8];
    load_run(w, a.w, a.w_bf16, c, n);
    double acc[8] = {};
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float rstd = a.rstd[row], mean = means[row];
        float h[8], d[8], dh[8] = {};
        load_run(h, a.h, a.h_bf16, row * a.ldh + c, n);
        load_run(d, a.dy, a.dy_bf16, row * a.lddy + c, n);
        if (a.dh) load_run(dh, a.dh, a.h_bf16, row * a.lddh + c, n);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float x = h[j] * rstd;
            acc[j] = __builtin_fma((double)d[j], (double)x, acc[j]);
            dh[j] += rstd * (d[j] * w[j] - x * mean);
        }
        store_run(dh, a.dx, a.h_bf16, row * a.lddx + c, n);
    }
    if (!part) return;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)acc[j];
    store_run(v, part, 0, blockIdx.y * a.cols + c, n);
}

// dw of 32 columns: 16 lanes a column take every 16th part
__global__ __launch_bounds__(512) void rmsnorm_grad_join_kernel(const float *part, int64_t parts, int64_t cols, float *dw)
{
    __shared__ double sums[16][33];
    const int col = threadIdx.x & 31, sub = threadIdx.x >> 5;
    const int64_t c = blockIdx.x * (int64_t)32 + col;
    double s = 0.0;
    if (c < cols) {
#pragma unroll 8
        for (int64_t i = sub; i < parts; i += 16) s += part[i * cols + c];
    }
    sums[sub][col] = s;
    __syncthreads();
    if (sub == 0 && c < cols) {
        for (int i = 1; i < 16; ++i) s += sums[i][col];
        dw[c] = (float)s;
    }
}

inline int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

// bytes that the cache may still hold from the kernels before: above, rows are read past it (16384 x
// 4096 bfloat16 101 -> 89 us; 8192 x 1024, which it holds, 18.8 -> 20.9)
constexpr int64_t kCached = int64_t(192) << 20;

constexpr int64_t kLong = 16384;       // columns that a workgroup's registers hold

// rows that a workgroup has at a time
int64_t rows_at_once(int64_t cols) { return cols <= 256 ? 16 : cols <= 1024 ? 4 : 1; }

// waves of a workgroup
int64_t waves_of(int64_t cols) { return cols <= 1024 ? 4 : cols <= 8192 ? (cols + 511) / 512 : (cols + 1023) / 1024; }

// workgroups, each with one part of dw
int64_t parts_of(int64_t rows, int64_t cols)
{
    if (cols > kLong) {
        // (the parts' memory stays at 128 MB where rows are very long)
        const int64_t fit = (int64_t(1) << 25) / cols, most = fit < 8 ? 8 : fit > 256 ? 256 : fit;
        return rows < most ? rows : most;
    }
    // as many as are there at once (registers: 16 waves a CU, 8 of those with several rows), each
    // with equally many turns: with twice as many 16384 x 4096 took 104 us instead of 102, 777 x 2049 15.1
    // instead of 12.6, with three quarters of them the first 113
    const int64_t most = 256 * (cols <= 1024 ? 2 : waves_of(cols) < 16 ? 16 / waves_of(cols) : 1);
    const int64_t per = rows_at_once(cols), groups = (rows + per - 1) / per, turns = (groups + most - 1) / most;
    return turns == 0 ? 0 : (groups + turns - 1) / turns;
}

int64_t means_bytes(int64_t rows, int64_t cols) { return cols > kLong ? up256(rows * 4) : 0; }

template <bool HB, bool DB, bool ONCE>
hipError_t launch_grad(const NormGradArgs &a, unsigned parts, float *part, hipStream_t s)
{
    constexpr int M = HB ? 1 : 2;           // chunks of 8 elements
    const dim3 grid(parts), block((unsigned)(64 * waves_of(a.cols)));
    if (a.cols <= 256) hipLaunchKernelGGL((rmsnorm_grad_kernel<HB, DB, 16, 2 * M, ONCE>), grid, block, 0, s, a, part);
    else if (a.cols <= 1024) hipLaunchKernelGGL((rmsnorm_grad_kernel<HB, DB, 64, 2 * M, ONCE>), grid, block, 0, s, a, part);
    else if (a.cols <= 8192) hipLaunchKernelGGL((rmsnorm_grad_kernel<HB, DB, 0, M, ONCE>), grid, block, 0, s, a, part);
    else hipLaunchKernelGGL((rmsnorm_grad_kernel<HB, DB, 0, 2 * M, ONCE>), grid, block, 0, s, a, part);
    return hipGetLastError();
}

template <bool HB, bool DB>
hipError_t launch_types(const NormGradArgs &a, unsigned parts, float *part, hipStream_t s)
{
    const int64_t bytes = a.rows * a.cols * ((a.dh ? 2 : 1) * (HB ? 2 : 4) + (DB ? 2 : 4));
    return bytes > kCached ? launch_grad<HB, DB, true>(a, parts, part, s) : launch_grad<HB, DB, false>(a, parts, part, s);
}

}  // namespace

int64_t rmsnorm_grad_workspace(int64_t rows, int64_t cols)
{
    return means_bytes(rows, cols) + up256(parts_of(rows, cols) * cols * 4);
}

hipError_t launch_rmsnorm_grad(const NormGradArgs &a, hipStream_t stream)
{
    const int64_t parts = parts_of(a.rows, a.cols);
    float *means = reinterpret_cast<float *>(a.workspace);
    float *sums = reinterpret_cast<float *>(a.workspace + means_bytes(a.rows, a.cols)), *part = a.dw ? sums : nullptr;
    if (a.rows > 0) {
        hipError_t e;
        if (a.cols > kLong) {
            hipLaunchKernelGGL(rmsnorm_grad_means_kernel, row_grid(a.rows), dim3(1024), 0, stream, a, means);
            hipLaunchKernelGGL(rmsnorm_grad_tile_kernel, dim3((unsigned)((a.cols + 2047) / 2048), (unsigned)parts), dim3(256), 0, stream, a, means, part);
            e = hipGetLastError();
        } else if (a.h_bf16) {
            e = a.dy_bf16 ? launch_types<true, true>(a, (unsigned)parts, part, stream) : launch_types<true, false>(a, (unsigned)parts, part, stream);
        } else {
            e = a.dy_bf16 ? launch_types<false, true>(a, (unsigned)parts, part, stream) : launch_types<false, false>(a, (unsigned)parts, part, stream);
        }
        if (e != hipSuccess) return e;
    }
    if (a.dw) hipLaunchKernelGGL(rmsnorm_grad_join_kernel, dim3((unsigned)((a.cols + 31) / 32)), dim3(512), 0, stream, sums, parts, a.cols, a.dw);
    return hipGetLastError();
}

}  // namespace q2d
