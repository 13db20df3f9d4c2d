// Root-mean-square norm of rows, with the residual's addition.
#include "norm_common.hpp"
#include "norms.hpp"

namespace q2d {

namespace {

__global__ __launch_bounds__(256) void rmsnorm_rows_kernel(const NormArgs a)
{
    __shared__ double lds[4];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t x0 = row * a.ldx, r0 = row * a.ldr, h0 = row * a.ldh, y0 = row * a.ldy;
        auto h_at = [&](int64_t c) __attribute__((always_inline)) {
            float v = load_value(a.x, a.x_bf16, x0 + c);
            if (a.r) {
                v += load_value(a.r, a.r_bf16, r0 + c);
                if (a.x_bf16) v = bf16_to_f(f_to_bf16_rne(v));
            }
            return v;
        };
        double s = 0.0;
        for (int64_t c = threadIdx.x; c < a.cols; c += 256) {
            const double v = h_at(c);
            s += v * v;
        }
        const float rstd = rstd_of(group_sum(s, 4, lds), a.cols, a.eps);
        if (threadIdx.x == 0) a.rstd[row] = rstd;
        for (int64_t c = threadIdx.x; c < a.cols; c += 256) {
            const float v = h_at(c);
            if (a.h) store_value(a.h, a.x_bf16, h0 + c, v);
            if (a.y) store_value(a.y, a.y_bf16, y0 + c, (v * rstd) * load_value(a.w, a.w_bf16, c));
        }
    }
}

}  // namespace

hipError_t launch_rmsnorm_rows(const NormArgs &a, hipStream_t stream)
{
    const int64_t most = 1 << 20;
    hipLaunchKernelGGL(rmsnorm_rows_kernel, dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace q2d
