// Gradient of the root-mean-square norm.
#include "norm_common.hpp"
#include "norms.hpp"
#include "kernels.hpp"

namespace q2d {

namespace {

// c = mean(dy * w * h) * rstd of each row
__global__ __launch_bounds__(256) void rmsnorm_grad_rows_kernel(const NormGradArgs a, float *means)
{
    __shared__ double lds[4];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float rstd = a.rstd[row];
        double s = 0.0;
        for (int64_t c = threadIdx.x; c < a.cols; c += 256)
            s += (load_value(a.dy, a.dy_bf16, row * a.lddy + c) * load_value(a.w, a.w_bf16, c)) *
                 (load_value(a.h, a.h_bf16, row * a.ldh + c) * rstd);
        s = group_sum(s, 4, lds);
        if (threadIdx.x == 0) means[row] = (float)(s / (double)a.cols);
    }
}

// 256 columns of every gridDim.y-th row: dx, and the sum of dy * xhat over these rows
__global__ __launch_bounds__(256) void rmsnorm_grad_tile_kernel(const NormGradArgs a, const float *means, float *part)
{
    const int64_t c = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (c >= a.cols) return;
    const float w = load_value(a.w, a.w_bf16, c);
    float sum = 0.f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float rstd = a.rstd[row];
        const float xh = load_value(a.h, a.h_bf16, row * a.ldh + c) * rstd;
        const float dy = load_value(a.dy, a.dy_bf16, row * a.lddy + c);
        float dx = rstd * (dy * w - xh * means[row]);
        if (a.dh) dx += load_value(a.dh, a.h_bf16, row * a.lddh + c);
        store_value(a.dx, a.h_bf16, row * a.lddx + c, dx);
        sum += dy * xh;
    }
    if (a.dw) part[blockIdx.y * a.cols + c] = sum;
}

__global__ __launch_bounds__(256) void rmsnorm_grad_join_kernel(const float *part, int64_t parts, int64_t cols, float *dw)
{
    const int64_t c = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (c >= cols) return;
    double s = 0.0;
    for (int64_t i = 0; i < parts; ++i) s += part[i * cols + c];
    dw[c] = (float)s;
}

int64_t parts_of(int64_t rows) { return rows < 256 ? rows : 256; }

inline int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

}  // namespace

int64_t rmsnorm_grad_workspace(int64_t rows, int64_t cols)
{
    return up256(rows * 4) + up256(parts_of(rows) * cols * 4);
}

hipError_t launch_rmsnorm_grad(const NormGradArgs &a, hipStream_t stream)
{
    const unsigned tiles = (unsigned)((a.cols + 255) / 256);
    float *means = reinterpret_cast<float *>(a.workspace), *part = reinterpret_cast<float *>(a.workspace + up256(a.rows * 4));
    const int64_t parts = parts_of(a.rows);
    if (a.rows > 0) {
        const int64_t most = 1 << 20;
        hipLaunchKernelGGL(rmsnorm_grad_rows_kernel, dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(256), 0, stream, a, means);
        hipLaunchKernelGGL(rmsnorm_grad_tile_kernel, dim3(tiles, (unsigned)parts), dim3(256), 0, stream, a, means, part);
    }
    if (a.dw) hipLaunchKernelGGL(rmsnorm_grad_join_kernel, dim3(tiles), dim3(256), 0, stream, part, parts, a.cols, a.dw);
    return hipGetLastError();
}

}  // namespace q2d
