// Launch interface of the root-mean-square norm and of the gradients' norm (host and device side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace q2d {

// One pass over rows: h = x + r (or x), rstd, and y = norm(h) * w.  Row r of a tensor starts
// at its pointer + r * ld elements.
struct NormArgs {
    const void *x; int64_t ldx;
    const void *r; int64_t ldr;        // or null
    const void *w;
    void *h;       int64_t ldh;        // set with r
    void *y;       int64_t ldy;        // or null
    float *rstd;
    int64_t rows, cols;
    double eps;
    int x_bf16, r_bf16, w_bf16, y_bf16;
};

hipError_t launch_rmsnorm_rows(const NormArgs &a, hipStream_t stream);

// Buffers of one quantized operand (null: not wanted)
struct QuantOut {
    uint8_t *codes;    int64_t ld_codes;
    uint8_t *codes_t;  int64_t ld_codes_t;
    uint8_t *scales;   int64_t ld_scales;
    uint8_t *scales_t; int64_t ld_scales_t;
};

// Operands of norm(h) * w, from h and its rows' rstd.
struct NormQuantArgs {
    const void *h; int64_t ldh;
    const float *rstd;
    const void *w;
    int64_t rows, cols, rows_pad, cols_pad;
    int h_bf16, w_bf16;
    int fp4;                           // 0 none, 1 2D blocks, 2 1D blocks
    int mx;
    int block;                         // edge of the 2D blocks
    QuantOut q4, q8;
};

hipError_t launch_rmsnorm_quantize(const NormQuantArgs &a, hipStream_t stream);

struct NormGradArgs {
    const void *h;  int64_t ldh;
    const void *dy; int64_t lddy;
    const void *dh; int64_t lddh;      // or null
    void *dx;       int64_t lddx;      // h's type, as dh
    const void *w;
    const float *rstd;
    float *dw;                         // or null
    int64_t rows, cols;
    int h_bf16, w_bf16, dy_bf16;
    uint8_t *workspace;
};

// bytes of workspace of a gradient of these sizes
int64_t rmsnorm_grad_workspace(int64_t rows, int64_t cols);
hipError_t launch_rmsnorm_grad(const NormGradArgs &a, hipStream_t stream);

}  // namespace q2d
