// Root-mean-square norm of rows, with the residual's addition.
//
// One read of x and the residual: a row stays in registers between the sum of its squares and
// the products with it.  A lane holds CH chunks of 16 bytes of x, chunk k of a row in lane k % (lanes
// of the row).  The squares are summed in 64 bits,
// where those of any float32 neither overflow nor vanish; the vector unit has time for it beside
// the memory, which bounds the kernel: 16384 x 4096, float32 with a bfloat16 residual, 134 us (805
// MB, 6.0 TB/s); bfloat16 86 us (6.2 TB/s); 777 x 2049 7 us, a single row 3.5, which is latency.
// Before, a workgroup a row and element by element from memory twice, the first took 378 us.
#include "norm_common.hpp"
#include "norms.hpp"

namespace q2d {

namespace {

// XB: x is bfloat16.  RT: no residual, a float32 or a bfloat16 one.  LANES: of a row: 16 or 64
// (a workgroup of 256 takes several rows), or 0 for all of the workgroup.  ONCE: x and the residual
// come from memory rather than from the cache.
template <bool XB, int RT, int LANES, int CH, bool ONCE>
__global__ __launch_bounds__(LANES ? 256 : 1024) void rmsnorm_rows_kernel(const NormArgs a)
{
    constexpr int EX = XB ? 2 : 4, ER = RT == 2 ? 2 : 4, N = 16 / EX;
    const int t = LANES ? threadIdx.x % (LANES ? LANES : 1) : threadIdx.x, step = LANES ? LANES : blockDim.x;
    const int64_t row = LANES ? group_index() * (256 / (LANES ? LANES : 1)) + threadIdx.x / (LANES ? LANES : 1) : group_index();
    if (LANES == 0 && row >= a.rows) return;
    // (lanes of a row beyond the last one hold nothing)
    const int64_t cols = row < a.rows ? a.cols : 0;
    const uint8_t *x = reinterpret_cast<const uint8_t *>(a.x) + row * a.ldx * EX;
    const uint8_t *r = reinterpret_cast<const uint8_t *>(a.r) + row * a.ldr * ER;
    Run<XB, N> h[CH];
    double sum = 0.0;
    {
        Run<RT == 2, N> d[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t c = N * (t + k * (int64_t)step);
            h[k].template load<ONCE>(x + c * EX, cols - c);
            if constexpr (RT != 0) d[k].template load<ONCE>(r + c * ER, cols - c);
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if constexpr (RT != 0) {
                float v[N];
#pragma unroll
                for (int j = 0; j < N; ++j) v[j] = h[k].at(j) + d[k].at(j);
                h[k].set(v);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const double v = h[k].at(j);
                sum = __builtin_fma(v, v, sum);
            }
        }
    }
    if constexpr (RT != 0) {
        uint8_t *out = reinterpret_cast<uint8_t *>(a.h) + row * a.ldh * EX;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t c = N * (t + k * (int64_t)step);
            h[k].store(out + c * EX, cols - c);
        }
    }
    if constexpr (LANES) {
        sum = lane_sum<LANES ? LANES : 64>(sum);
    } else {
        __shared__ double lds[16];
        sum = group_sum(sum, blockDim.x >> 6, lds);
    }
    const float rstd = rstd_of(sum, a.cols, a.eps);
    if (t == 0 && row < a.rows) a.rstd[row] = rstd;
    if (!a.y) return;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int64_t c = N * (t + k * (int64_t)step);
        if (c >= cols) break;
        float w[N], y[N];
        load_run(w, a.w, a.w_bf16, c, cols - c);
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = (h[k].at(j) * rstd) * w[j];
        store_run(y, a.y, a.y_bf16, row * a.ldy + c, cols - c);
    }
}

// Rows that no workgroup's registers hold: a second read of what this lane read or wrote
__global__ __launch_bounds__(1024) void rmsnorm_long_rows_kernel(const NormArgs a)
{
    const int64_t row = group_index();
    if (row >= a.rows) return;
    double sum = 0.0;
    for (int64_t c = 8 * (int64_t)threadIdx.x; c < a.cols; c += 8 * 1024) {
        float v[8], d[8];
        load_run(v, a.x, a.x_bf16, row * a.ldx + c, a.cols - c);
        if (a.r) {
            load_run(d, a.r, a.r_bf16, row * a.ldr + c, a.cols - c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] += d[j];
                if (a.x_bf16) v[j] = round_bf16(v[j]);
            }
            store_run(v, a.h, a.x_bf16, row * a.ldh + c, a.cols - c);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = __builtin_fma((double)v[j], (double)v[j], sum);
    }
    __shared__ double lds[16];
    const float rstd = rstd_of(group_sum(sum, 16, lds), a.cols, a.eps);
    if (threadIdx.x == 0) a.rstd[row] = rstd;
    if (!a.y) return;
    const void *h = a.r ? a.h : a.x;
    const int64_t ldh = a.r ? a.ldh : a.ldx;
    for (int64_t c = 8 * (int64_t)threadIdx.x; c < a.cols; c += 8 * 1024) {
        float v[8], w[8];
        load_run(v, h, a.x_bf16, row * ldh + c, a.cols - c);
        load_run(w, a.w, a.w_bf16, c, a.cols - c);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (v[j] * rstd) * w[j];
        store_run(v, a.y, a.y_bf16, row * a.ldy + c, a.cols - c);
    }
}

// `per` rows a workgroup.  (Work-items along one dimension of a launch stay below 2^32: rows beyond
// 2^20 workgroups go along the second.)
template <bool XB, int RT, int LANES, int CH, bool ONCE>
hipError_t launch_c(const NormArgs &a, int64_t per, unsigned threads, hipStream_t s)
{
    hipLaunchKernelGGL((rmsnorm_rows_kernel<XB, RT, LANES, CH, ONCE>), row_grid((a.rows + per - 1) / per), dim3(threads), 0, s, a);
    return hipGetLastError();
}

// Inputs larger than the cache are read past it, so that it keeps more of h for the next kernel:
// 16384 x 4096 bfloat16 95 -> 83 us, with operands in FP4 and MXFP8 148 -> 132.  Not narrow rows,
// which share lines (100000 x 200 35 us instead of 31).
constexpr int64_t kCached = int64_t(192) << 20;

template <bool XB, int RT>
hipError_t launch_r(const NormArgs &a, hipStream_t s)
{
    constexpr int N = XB ? 8 : 4, M = 8 / N;            // elements of a chunk, chunks of 8 elements
    const int64_t bytes = a.rows * a.cols * ((XB ? 2 : 4) + (RT == 0 ? 0 : RT == 1 ? 4 : 2));
    const bool once = bytes > kCached;
    if (a.cols <= 256) return launch_c<XB, RT, 16, 2 * M, false>(a, 16, 256, s);
    if (a.cols <= 1024) return once ? launch_c<XB, RT, 64, 2 * M, true>(a, 4, 256, s) : launch_c<XB, RT, 64, 2 * M, false>(a, 4, 256, s);
    // 16 elements a lane, 8 of float32 (16384 x 4096 149 us with 16), 32 of long rows
    const auto threads = [&](int ch) { return (unsigned)((a.cols + 64 * N * ch - 1) / (64 * N * ch) * 64); };
    if (a.cols <= 8192)
        return once ? launch_c<XB, RT, 0, 2, true>(a, 1, threads(2), s) : launch_c<XB, RT, 0, 2, false>(a, 1, threads(2), s);
    if (a.cols <= 16384)
        return once ? launch_c<XB, RT, 0, 2 * M, true>(a, 1, threads(2 * M), s) : launch_c<XB, RT, 0, 2 * M, false>(a, 1, threads(2 * M), s);
    return once ? launch_c<XB, RT, 0, 4 * M, true>(a, 1, threads(4 * M), s) : launch_c<XB, RT, 0, 4 * M, false>(a, 1, threads(4 * M), s);
}

}  // namespace

hipError_t launch_rmsnorm_rows(const NormArgs &a, hipStream_t stream)
{
    if (a.cols > 32768) {
        hipLaunchKernelGGL(rmsnorm_long_rows_kernel, row_grid(a.rows), dim3(1024), 0, stream, a);
        return hipGetLastError();
    }
    const int rt = !a.r ? 0 : a.r_bf16 ? 2 : 1;
    if (a.x_bf16) return rt == 0 ? launch_r<true, 0>(a, stream) : rt == 1 ? launch_r<true, 1>(a, stream) : launch_r<true, 2>(a, stream);
    return rt == 0 ? launch_r<false, 0>(a, stream) : rt == 1 ? launch_r<false, 1>(a, stream) : launch_r<false, 2>(a, stream);
}

}  // namespace q2d
