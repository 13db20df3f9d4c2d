// Layout arithmetic and argument checks that the entry points share (host only).
#pragma once

#include "q2d.h"

#include <stdint.h>

namespace q2d {

constexpr int64_t kPadK = 128;     // K extents are padded to the GEMM K-tile

inline int64_t rup(int64_t a, int64_t m) { return (a + m - 1) / m * m; }
inline int64_t cdiv(int64_t a, int64_t m) { return (a + m - 1) / m; }
inline bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) % n) == 0; }

struct Layout {
    int64_t ld_codes, ld_codes_t, ld_scales, ld_scales_t;
    int64_t rows_codes, rows_codes_t, rows_scales, rows_scales_t;
};

inline Layout layout_of(q2d_fmt fmt, int64_t R, int64_t C)
{
    Layout l;
    if (fmt == Q2D_FMT_FP4_2D) {
        l.ld_codes = rup(C, kPadK) / 2;   l.rows_codes = R;
        l.ld_codes_t = rup(R, kPadK) / 2; l.rows_codes_t = C;
        l.ld_scales = rup(C, kPadK) / 32; l.rows_scales = cdiv(R, 32);
        l.ld_scales_t = rup(R, kPadK) / 32; l.rows_scales_t = cdiv(C, 32);
    } else if (fmt == Q2D_FMT_FP4_1D) {
        // scales: one 4-byte word per row and K-tile, K-tile major
        l.ld_codes = rup(C, kPadK) / 2;   l.rows_codes = R;
        l.ld_codes_t = rup(R, kPadK) / 2; l.rows_codes_t = C;
        l.ld_scales = 4 * R;              l.rows_scales = rup(C, kPadK) / kPadK;
        l.ld_scales_t = 4 * C;            l.rows_scales_t = rup(R, kPadK) / kPadK;
    } else {
        l.ld_codes = rup(C, kPadK);       l.rows_codes = R;
        l.ld_codes_t = rup(R, kPadK);     l.rows_codes_t = C;
        l.ld_scales = rup(C, kPadK) / 32; l.rows_scales = R;
        l.ld_scales_t = rup(R, kPadK) / 32; l.rows_scales_t = C;
    }
    return l;
}

inline bool valid_dtype(q2d_dtype d) { return d == Q2D_F32 || d == Q2D_BF16; }
inline int dtype_bytes(q2d_dtype d) { return d == Q2D_F32 ? 4 : 2; }

// Check one orientation's buffers against the minimal layout.
inline bool check_pair(const uint8_t *codes, int64_t ldc, int64_t min_ldc, const uint8_t *scales,
                int64_t lds, int64_t min_lds)
{
    if (!codes) return true;
    if (!scales) return false;
    if (ldc < min_ldc || (ldc % 16) != 0 || lds < min_lds || (lds % 4) != 0) return false;
    return aligned(codes, 16) && aligned(scales, 4);
}

inline q2d_status check_tensor(const q2d_tensor *t, q2d_fmt fmt, int64_t R, int64_t C)
{
    if (!t) return Q2D_EINVAL;
    if (t->fmt != fmt || t->rows != R || t->cols != C) return Q2D_EINVAL;
    if (t->block != 32 && !(t->block == 64 && fmt == Q2D_FMT_FP4_2D)) return Q2D_EUNSUPPORTED;
    if (!t->codes && !t->codes_t) return Q2D_EINVAL;
    const Layout l = layout_of(fmt, R, C);
    if (!check_pair(t->codes, t->ld_codes, l.ld_codes, t->scales, t->ld_scales, l.ld_scales)) return Q2D_EINVAL;
    if (!check_pair(t->codes_t, t->ld_codes_t, l.ld_codes_t, t->scales_t, t->ld_scales_t, l.ld_scales_t))
        return Q2D_EINVAL;
    return Q2D_OK;
}

// Matrix extents: positive, and at most 2^31 per dimension, which keeps every
// layout product and padded size far from int64 overflow.
constexpr int64_t kMaxDim = int64_t(1) << 31;

inline q2d_status check_dims(int64_t R, int64_t C)
{
    if (R <= 0 || C <= 0) return Q2D_EINVAL;
    if (R > kMaxDim || C > kMaxDim) return Q2D_EUNSUPPORTED;
    return Q2D_OK;
}

// 128 x 256 tiles of one launch, in a grid of two dimensions: 2^20 along the first, 2^15 along the second
constexpr int64_t kMaxTiles = int64_t(1) << 35;

inline bool few_tiles(int64_t R, int64_t C) { return cdiv(R, 128) * cdiv(C, 256) <= kMaxTiles; }

}  // namespace q2d
