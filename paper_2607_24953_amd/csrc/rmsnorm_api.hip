// C ABI of the root-mean-square norm: argument validation and launches.
#include "q2d.h"
#include "layout.hpp"
#include "norms.hpp"

#include <math.h>

namespace {

using namespace q2d;

constexpr int64_t kMaxIndex = int64_t(1) << 47;
constexpr int64_t kMaxRows = INT32_MAX, kMaxCols = int64_t(1) << 27;

// A tensor's rows in memory, in bytes
struct Rows {
    uintptr_t at = 0;
    int64_t rows = 0, width = 0, pitch = 0;
    uintptr_t end() const { return at + (uintptr_t)((rows - 1) * pitch + width); }
};

// whether no byte belongs to both
bool apart(const Rows &a, const Rows &b)
{
    if (!a.at || !b.at || a.rows <= 0 || b.rows <= 0 || a.end() <= b.at || b.end() <= a.at) return true;
    // rows of one pitch side by side in one buffer
    if (a.pitch != b.pitch || a.rows == 1 || b.rows == 1) return false;
    const int64_t p = a.pitch, d = (((int64_t)b.at - (int64_t)a.at) % p + p) % p;
    return a.width <= d && d + b.width <= p;
}

bool same(const Rows &a, const Rows &b) { return a.at == b.at && a.rows == b.rows && a.width == b.width && (a.pitch == b.pitch || a.rows == 1); }

// Rows of `cols` elements, which do not share memory with one another
q2d_status check_rows(const void *p, int32_t dt, int64_t rows, int64_t cols, int64_t ld, Rows *out)
{
    if (!valid_dtype((q2d_dtype)dt)) return Q2D_EINVAL;
    if (rows == 0) return Q2D_OK;                  // (no memory, no address)
    if (!p) return Q2D_EINVAL;
    const int64_t size = dtype_bytes((q2d_dtype)dt);
    if (!aligned(p, (uintptr_t)size)) return Q2D_EINVAL;
    if (rows > 1 && ld < cols) return Q2D_EINVAL;
    int64_t last = cols;
    if (rows > 1 && (__builtin_mul_overflow(rows - 1, ld, &last) || __builtin_add_overflow(last, cols, &last))) return Q2D_EUNSUPPORTED;
    if (last >= kMaxIndex) return Q2D_EUNSUPPORTED;
    *out = {reinterpret_cast<uintptr_t>(p), rows, cols * size, rows > 1 ? ld * size : cols * size};
    return Q2D_OK;
}

Rows vector_of(const void *p, int64_t n, int64_t size) { return {reinterpret_cast<uintptr_t>(p), 1, n * size, n * size}; }

// Buffers of a quantized operand, as memory that the call writes
int buffers_of(const q2d_tensor *t, Rows out[4])
{
    const Layout l = layout_of((q2d_fmt)t->fmt, t->rows, t->cols);
    int n = 0;
    if (t->codes) {
        out[n++] = vector_of(t->codes, l.rows_codes, t->ld_codes);
        out[n++] = vector_of(t->scales, l.rows_scales, t->ld_scales);
    }
    if (t->codes_t) {
        out[n++] = vector_of(t->codes_t, l.rows_codes_t, t->ld_codes_t);
        out[n++] = vector_of(t->scales_t, l.rows_scales_t, t->ld_scales_t);
    }
    return n;
}

QuantOut out_of(const q2d_tensor *t)
{
    return {t->codes, t->ld_codes, t->codes_t, t->ld_codes_t, t->scales, t->ld_scales, t->scales_t, t->ld_scales_t};
}

}  // namespace

extern "C" {

q2d_status q2d_rmsnorm_fwd(const q2d_rmsnorm *n, q2d_tensor *q4, q2d_tensor *q8, hipStream_t stream)
{
    if (!n || n->rows < 0 || n->cols <= 0) return Q2D_EINVAL;
    if (n->rows > kMaxRows || n->cols > kMaxCols) return Q2D_EUNSUPPORTED;
    // (eps within float32's normal numbers: 1 / sqrt(eps) stays below 2^63)
    if (!(n->eps >= 0x1p-126) || !std::isfinite(n->eps)) return Q2D_EINVAL;
    if (!valid_dtype((q2d_dtype)n->weight_dtype) || !n->weight || !aligned(n->weight, dtype_bytes((q2d_dtype)n->weight_dtype))) return Q2D_EINVAL;
    if (n->rows && (!n->residual != !n->h)) return Q2D_EINVAL;
    if (!aligned(n->rstd, 4)) return Q2D_EINVAL;
    if (n->rows == 0 ? q4 || q8 : (!n->y && !q4 && !q8) || !n->rstd) return Q2D_EINVAL;
    Rows x, r, h, y;
    q2d_status s = check_rows(n->x, n->x_dtype, n->rows, n->cols, n->ldx, &x);
    if (s == Q2D_OK && n->residual) s = check_rows(n->residual, n->residual_dtype, n->rows, n->cols, n->ld_residual, &r);
    if (s == Q2D_OK && n->h) s = check_rows(n->h, n->x_dtype, n->rows, n->cols, n->ldh, &h);
    if (s == Q2D_OK && n->y) s = check_rows(n->y, n->y_dtype, n->rows, n->cols, n->ldy, &y);
    if (s == Q2D_OK && q4) {
        if (q4->fmt != Q2D_FMT_FP4_2D && q4->fmt != Q2D_FMT_FP4_1D) return Q2D_EINVAL;
        s = check_tensor(q4, (q2d_fmt)q4->fmt, n->rows, n->cols);
    }
    if (s == Q2D_OK && q8) s = check_tensor(q8, Q2D_FMT_MXFP8, n->rows, n->cols);
    if (s == Q2D_OK && (q4 || q8) && !few_tiles(n->rows, n->cols)) return Q2D_EUNSUPPORTED;
    if (s != Q2D_OK) return s;

    // what is written meets nothing else, but that h may take the place of x or of the residual
    Rows out[3 + 8] = {h, y, vector_of(n->rstd, n->rows, 4)};
    int outs = 3;
    if (q4) outs += buffers_of(q4, out + outs);
    if (q8) outs += buffers_of(q8, out + outs);
    const Rows w = vector_of(n->weight, n->cols, dtype_bytes((q2d_dtype)n->weight_dtype));
    for (int i = 0; i < outs; ++i) {
        for (int j = 0; j < i; ++j)
            if (!apart(out[i], out[j])) return Q2D_EINVAL;
        const bool stream_out = i == 0;
        if (!apart(out[i], w)) return Q2D_EINVAL;
        if (!apart(out[i], x) && !(stream_out && same(out[i], x))) return Q2D_EINVAL;
        if (!apart(out[i], r) && !(stream_out && same(out[i], r) && n->residual_dtype == n->x_dtype)) return Q2D_EINVAL;
    }
    if (n->rows == 0) return Q2D_OK;

    NormArgs a;
    a.x = n->x; a.ldx = n->ldx;
    a.r = n->residual; a.ldr = n->ld_residual;
    a.w = n->weight;
    a.h = n->h; a.ldh = n->ldh;
    a.y = n->y; a.ldy = n->ldy;
    a.rstd = n->rstd;
    a.rows = n->rows; a.cols = n->cols; a.eps = n->eps;
    a.x_bf16 = n->x_dtype == Q2D_BF16; a.r_bf16 = n->residual_dtype == Q2D_BF16;
    a.w_bf16 = n->weight_dtype == Q2D_BF16; a.y_bf16 = n->y_dtype == Q2D_BF16;
    if (launch_rmsnorm_rows(a, stream) != hipSuccess) return Q2D_ELAUNCH;
    if (!q4 && !q8) return Q2D_OK;

    NormQuantArgs b = {};
    b.h = n->h ? n->h : n->x;
    b.ldh = n->rows == 1 ? n->cols : n->h ? n->ldh : n->ldx;
    b.rstd = n->rstd; b.w = n->weight;
    b.rows = n->rows; b.cols = n->cols;
    b.rows_pad = rup(n->rows, 128); b.cols_pad = rup(n->cols, 128);
    b.h_bf16 = a.x_bf16; b.w_bf16 = a.w_bf16;
    b.fp4 = !q4 ? 0 : q4->fmt == Q2D_FMT_FP4_2D ? 1 : 2;
    b.mx = q8 != nullptr;
    b.block = 32;
    if (q4) { b.q4 = out_of(q4); b.block = q4->block; }
    if (q8) b.q8 = out_of(q8);
    return launch_rmsnorm_quantize(b, stream) == hipSuccess ? Q2D_OK : Q2D_ELAUNCH;
}

int64_t q2d_rmsnorm_workspace(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols <= 0 || rows > kMaxRows || cols > kMaxCols) return -1;
    return rmsnorm_grad_workspace(rows, cols);
}

q2d_status q2d_rmsnorm_bwd(const q2d_rmsnorm_grad *n, void *workspace, int64_t workspace_bytes, hipStream_t stream)
{
    if (!n || n->rows < 0 || n->cols <= 0) return Q2D_EINVAL;
    if (n->rows > kMaxRows || n->cols > kMaxCols) return Q2D_EUNSUPPORTED;
    if (!valid_dtype((q2d_dtype)n->weight_dtype) || !n->weight || !aligned(n->weight, dtype_bytes((q2d_dtype)n->weight_dtype))) return Q2D_EINVAL;
    if ((n->rows && !n->rstd) || !aligned(n->rstd, 4) || !aligned(n->dw, 4)) return Q2D_EINVAL;
    Rows h, dy, dh, dx;
    q2d_status s = check_rows(n->h, n->h_dtype, n->rows, n->cols, n->ldh, &h);
    if (s == Q2D_OK) s = check_rows(n->dy, n->dy_dtype, n->rows, n->cols, n->lddy, &dy);
    if (s == Q2D_OK && n->dh) s = check_rows(n->dh, n->h_dtype, n->rows, n->cols, n->lddh, &dh);
    if (s == Q2D_OK) s = check_rows(n->dx, n->h_dtype, n->rows, n->cols, n->lddx, &dx);
    if (s != Q2D_OK) return s;
    const int64_t need = rmsnorm_grad_workspace(n->rows, n->cols);
    if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return Q2D_EINVAL;
    const Rows w = vector_of(n->weight, n->cols, dtype_bytes((q2d_dtype)n->weight_dtype)), rstd = vector_of(n->rstd, n->rows, 4);
    const Rows dw = vector_of(n->dw, n->cols, 4), ws = vector_of(workspace, 1, need);
    // dx may take the place of dh, or of dy where the types are the same
    const Rows *in[5] = {&h, &dy, &dh, &w, &rstd};
    for (int i = 0; i < 5; ++i) {
        const bool place = (i == 1 && n->dy_dtype == n->h_dtype) || i == 2;
        if (!apart(dw, *in[i]) || !apart(ws, *in[i])) return Q2D_EINVAL;
        if (!apart(dx, *in[i]) && !(place && same(dx, *in[i]))) return Q2D_EINVAL;
    }
    if (!apart(dx, dw) || !apart(dx, ws) || !apart(dw, ws)) return Q2D_EINVAL;

    NormGradArgs a;
    a.h = n->h; a.ldh = n->ldh;
    a.dy = n->dy; a.lddy = n->lddy;
    a.dh = n->dh; a.lddh = n->lddh;
    a.dx = n->dx; a.lddx = n->lddx;
    a.w = n->weight; a.rstd = n->rstd; a.dw = n->dw;
    a.rows = n->rows; a.cols = n->cols;
    a.h_bf16 = n->h_dtype == Q2D_BF16; a.w_bf16 = n->weight_dtype == Q2D_BF16; a.dy_bf16 = n->dy_dtype == Q2D_BF16;
    a.workspace = reinterpret_cast<uint8_t *>(workspace);
    return launch_rmsnorm_grad(a, stream) == hipSuccess ? Q2D_OK : Q2D_ELAUNCH;
}

}  // extern "C"
