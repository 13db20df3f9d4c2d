// Gradient of the root-mean-square norm.
//
// With n = h * rstd and g = dy * w: dx = rstd * (g - n * mean(g n)) + dh, dw = sum over rows of dy n.
// One read of h, dy and dh: a row stays in registers between the sum for its mean and the products
// with it, as in the forward kernel.  A workgroup takes every gridDim.x-th row and keeps its part
// of dw over all of them, in 64 bits: in registers, for rows of 4097 to 6144 and of 8193 to 16384 columns in
// LDS.  The parts lie one behind the other in the workspace and a second kernel adds them up.  Every
// sum has one owner and one order.
//
// The memory bounds it: 16384 x 4096 bfloat16 with dh 86 us (545 MB, 6.3 TB/s) and 5 for the join,
// float32 151 in all; 777 x 2049 8.5 + 3.5.  The statistics of a row and the products with it as two
// kernels, element by element, took 700.  Rows of more than 16384 columns are
// read twice (2048 x 17000 bfloat16 27 + 51 us); of 8193 to 16384 so 2048 x 12288 bfloat16 took 60 us,
// float32 101 (in registers, spilled, 77 and 165), with dw's parts in LDS 50 and 79 (4.0 and 5.1 TB/s): one
// workgroup has a CU for itself and nothing runs while it waits at its barrier.  With dw's parts in LDS for
// all rows, and six or eight waves to a SIMD, 16384 x 4096 took 103 and 102 us instead of 92.
//
// Rows of up to 1024 columns are further from that: the registers hold two waves a SIMD, each with one
// row at a time, and chunks that narrow rows leave empty stand for bytes that are not in flight.  bfloat16
// with dh: 65536 x 512 63 us (4.3 TB/s), 8192 x 1024 16 (from the cache), 100000 x 200 34 (4.7), 500000 x 128
// 110 (4.6), 500000 x 64 107 (2.4).
#include "norm_common.hpp"
#include "norms.hpp"
#include "kernels.hpp"

namespace q2d {

namespace {

// HB, DB: h and dh, dy are bfloat16.  LANES, CH: as in the forward kernel.  ONCE: the rows come from
// memory rather than from the cache.  FAR: 0, or the most lanes of a workgroup whose parts of dw are in
// LDS, each lane's own: two chunks' do not fit the registers of 16 waves, and without them two
// workgroups of 12 fit a CU.
template <bool HB, bool DB, int LANES, int CH, bool ONCE, int FAR = 0>
__global__ __launch_bounds__(LANES ? 256 : FAR ? FAR : 1024, LANES ? 1 : FAR == 768 ? 6 : 4) void rmsnorm_grad_kernel(const NormGradArgs a, float *part)
{
    constexpr int EH = HB ? 2 : 4, ED = DB ? 2 : 4, N = 16 / EH;
    constexpr int kPer = LANES ? 256 / (LANES ? LANES : 1) : 1;        // rows at a time
    __shared__ double lds[2][16];
    const int t = LANES ? threadIdx.x % (LANES ? LANES : 1) : threadIdx.x, step = LANES ? LANES : blockDim.x;
    const int sub = LANES ? threadIdx.x / (LANES ? LANES : 1) : 0;
    __shared__ double far[FAR ? CH * N : 1][FAR ? FAR : 1];
    float w[CH][N];
    double acc[FAR ? 1 : CH][FAR ? 1 : N];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int64_t c = N * (t + k * (int64_t)step);
        load_run(w[k], a.w, a.w_bf16, c, a.cols - c);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if constexpr (FAR) far[k * N + j][threadIdx.x] = 0.0;
            else acc[k][j] = 0.0;
        }
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
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float n = h[k].at(j) * rstd, d = dy[k].at(j);
                sum = __builtin_fma((double)(d * w[k][j]), (double)n, sum);
                if constexpr (FAR) far[k * N + j][threadIdx.x] = __builtin_fma((double)d, (double)n, far[k * N + j][threadIdx.x]);
                else acc[k][j] = __builtin_fma((double)d, (double)n, acc[k][j]);
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
            for (int j = 0; j < N; ++j) v[j] = (float)(FAR ? far[FAR ? k * N + j : 0][FAR ? threadIdx.x : 0] : acc[FAR ? 0 : k][FAR ? 0 : j]);
            o.set(v);
            o.store(reinterpret_cast<uint8_t *>(part + c), a.cols - c);
        }
    }
}

// Rows that no workgroup's registers hold: their means first
template <bool HB, bool DB>
__global__ __launch_bounds__(1024) void rmsnorm_grad_means_kernel(const NormGradArgs a, float *means)
{
    constexpr int EH = HB ? 2 : 4, ED = DB ? 2 : 4, N = 16 / EH;
    const int64_t row = group_index();
    if (row >= a.rows) return;
    __shared__ double lds[16];
    const uint8_t *hp = reinterpret_cast<const uint8_t *>(a.h) + row * a.ldh * EH;
    const uint8_t *dyp = reinterpret_cast<const uint8_t *>(a.dy) + row * a.lddy * ED;
    const float rstd = a.rstd[row];
    double s = 0.0;
#pragma unroll 2
    for (int64_t c = N * (int64_t)threadIdx.x; c < a.cols; c += N * 1024) {
        Run<HB, N> h;
        Run<DB, N> dy;
        float w[N];
        h.load(hp + c * EH, a.cols - c);
        dy.load(dyp + c * ED, a.cols - c);
        load_run(w, a.w, a.w_bf16, c, a.cols - c);
#pragma unroll
        for (int j = 0; j < N; ++j) s = __builtin_fma((double)(dy.at(j) * w[j]), (double)(h.at(j) * rstd), s);
    }
    s = group_sum(s, 16, lds);
    if (threadIdx.x == 0) means[row] = (float)(s / (double)a.cols);
}

// .. then 256 lanes' columns of every gridDim.y-th row, the last rows first: the cache may hold them
// still
template <bool HB, bool DB, bool ONCE>
__global__ __launch_bounds__(256) void rmsnorm_grad_tile_kernel(const NormGradArgs a, const float *means, float *part)
{
    constexpr int EH = HB ? 2 : 4, ED = DB ? 2 : 4, N = 16 / EH;
    const int64_t c = N * (blockIdx.x * (int64_t)256 + threadIdx.x), cols = a.cols - c;
    if (cols <= 0) return;
    float w[N];
    load_run(w, a.w, a.w_bf16, c, cols);
    double acc[N] = {};
    for (int64_t row = a.rows - 1 - blockIdx.y; row >= 0; row -= gridDim.y) {
        Run<HB, N> h, dh;
        Run<DB, N> dy;
        h.template load<ONCE>(reinterpret_cast<const uint8_t *>(a.h) + (row * a.ldh + c) * EH, cols);
        dy.template load<ONCE>(reinterpret_cast<const uint8_t *>(a.dy) + (row * a.lddy + c) * ED, cols);
        if (a.dh) dh.template load<ONCE>(reinterpret_cast<const uint8_t *>(a.dh) + (row * a.lddh + c) * EH, cols);
        else dh.zero();
        const float rstd = a.rstd[row], mean = means[row];
        float dx[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float n = h.at(j) * rstd, d = dy.at(j);
            acc[j] = __builtin_fma((double)d, (double)n, acc[j]);
            dx[j] = rstd * (d * w[j] - n * mean) + dh.at(j);
        }
        Run<HB, N> o;
        o.set(dx);
        o.store(reinterpret_cast<uint8_t *>(a.dx) + (row * a.lddx + c) * EH, cols);
    }
    if (!part) return;
    float v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = (float)acc[j];
    Run<false, N> o;
    o.set(v);
    o.store(reinterpret_cast<uint8_t *>(part + blockIdx.y * a.cols + c), cols);
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

// tiles of 256 lanes' columns
int64_t tiles_of(int64_t cols, bool h_bf16) { return (cols + (h_bf16 ? 2047 : 1023)) / (h_bf16 ? 2048 : 1024); }

// rows of nine to twelve waves: two workgroups to a CU with dw's parts in LDS (8192 x 5120 bfloat16
// 80 us, so 65, float32 105, 101; 2048 rows 26.5, 23.9, and 34.7, 32.4)
bool two_of_twelve(int64_t cols) { return cols > 4096 && cols <= 6144; }

// workgroups (of long rows: for each of their tiles), each with one part of dw
int64_t parts_of(int64_t rows, int64_t cols, bool h_bf16)
{
    if (cols > kLong) {
        // (1024 workgroups: with twice as many 8192 x 12288 float32 took 456 us instead of 434, with half
        // as many 2048 x 8448 bfloat16 49 instead of 45)
        const int64_t tiles = tiles_of(cols, h_bf16), most = tiles < 1024 ? 1024 / tiles : 1, turns = (rows + most - 1) / most;
        return turns == 0 ? 0 : (rows + turns - 1) / turns;
    }
    // as many as are there at once (registers: 16 waves a CU, 8 of those with several rows), each
    // with equally many turns: with twice as many 16384 x 4096 took 104 us instead of 102, 777 x 2049 15.1
    // instead of 12.6, with three quarters of them the first 113
    const int64_t most = 256 * (cols <= 1024 || two_of_twelve(cols) ? 2 : waves_of(cols) < 16 ? 16 / waves_of(cols) : 1);
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
    else if (two_of_twelve(a.cols)) hipLaunchKernelGGL((rmsnorm_grad_kernel<HB, DB, 0, M, ONCE, 768>), grid, block, 0, s, a, part);
    else if (a.cols <= 8192) hipLaunchKernelGGL((rmsnorm_grad_kernel<HB, DB, 0, M, ONCE>), grid, block, 0, s, a, part);
    else hipLaunchKernelGGL((rmsnorm_grad_kernel<HB, DB, 0, 2 * M, ONCE, 1024>), grid, block, 0, s, a, part);
    return hipGetLastError();
}

template <bool HB, bool DB>
hipError_t launch_types(const NormGradArgs &a, unsigned parts, float *means, float *part, hipStream_t s)
{
    const int64_t bytes = a.rows * a.cols * ((a.dh ? 2 : 1) * (HB ? 2 : 4) + (DB ? 2 : 4));
    if (a.cols > kLong) {
        hipLaunchKernelGGL((rmsnorm_grad_means_kernel<HB, DB>), row_grid(a.rows), dim3(1024), 0, s, a, means);
        const dim3 grid((unsigned)tiles_of(a.cols, HB), parts);
        if (bytes > kCached) hipLaunchKernelGGL((rmsnorm_grad_tile_kernel<HB, DB, true>), grid, dim3(256), 0, s, a, means, part);
        else hipLaunchKernelGGL((rmsnorm_grad_tile_kernel<HB, DB, false>), grid, dim3(256), 0, s, a, means, part);
        return hipGetLastError();
    }
    return bytes > kCached ? launch_grad<HB, DB, true>(a, parts, part, s) : launch_grad<HB, DB, false>(a, parts, part, s);
}

}  // namespace

int64_t rmsnorm_grad_workspace(int64_t rows, int64_t cols)
{
    // (bfloat16's are at least as many as float32's)
    return means_bytes(rows, cols) + up256(parts_of(rows, cols, true) * cols * 4);
}

hipError_t launch_rmsnorm_grad(const NormGradArgs &a, hipStream_t stream)
{
    const int64_t parts = parts_of(a.rows, a.cols, a.h_bf16);
    float *means = reinterpret_cast<float *>(a.workspace);
    float *sums = reinterpret_cast<float *>(a.workspace + means_bytes(a.rows, a.cols)), *part = a.dw ? sums : nullptr;
    if (a.rows > 0) {
        hipError_t e;
        if (a.h_bf16) {
            e = a.dy_bf16 ? launch_types<true, true>(a, (unsigned)parts, means, part, stream) : launch_types<true, false>(a, (unsigned)parts, means, part, stream);
        } else {
            e = a.dy_bf16 ? launch_types<false, true>(a, (unsigned)parts, means, part, stream) : launch_types<false, false>(a, (unsigned)parts, means, part, stream);
        }
        if (e != hipSuccess) return e;
    }
    if (a.dw) hipLaunchKernelGGL(rmsnorm_grad_join_kernel, dim3((unsigned)((a.cols + 31) / 32)), dim3(512), 0, stream, sums, parts, a.cols, a.dw);
    return hipGetLastError();
}

}  // namespace q2d
