// C ABI of the attention operators: argument validation, workspace layout and launches.
#include "q2d.h"
#include "attention.hpp"

#include <limits.h>
#include <math.h>

namespace {

using namespace q2d;

constexpr int64_t kMaxLen = int64_t(1) << 30;
constexpr int64_t kMaxPitch = int64_t(1) << 24;    // the tile loads' 32-bit row offsets

inline bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

// whole 16-byte rows, and a last element within 2^47
q2d_status check_heads(const q2d_heads &t, int64_t batch, int64_t length, int64_t heads, int64_t dim, int per)
{
    if (!t.data || !on16(t.data)) return Q2D_EINVAL;
    const int64_t n[3] = {batch, length, heads}, s[3] = {t.stride_batch, t.stride_length, t.stride_head};
    int64_t last = dim - 1;
    for (int i = 0; i < 3; ++i) {
        if (s[i] < 0 || (n[i] > 1 && s[i] % per != 0)) return Q2D_EINVAL;
        int64_t x;
        if (__builtin_mul_overflow(n[i] - 1, s[i], &x) || __builtin_add_overflow(last, x, &last) ||
            last >= (int64_t(1) << 47))
            return Q2D_EUNSUPPORTED;
    }
    if (length > 1 && t.stride_length >= kMaxPitch) return Q2D_EUNSUPPORTED;
    return Q2D_OK;
}

// (an output's rows must not share memory)
q2d_status check_output(const q2d_heads &t, int64_t batch, int64_t length, int64_t heads, int64_t dim, int per)
{
    const q2d_status s = check_heads(t, batch, length, heads, dim, per);
    if (s != Q2D_OK) return s;
    if ((batch > 1 && t.stride_batch < dim) || (length > 1 && t.stride_length < dim) || (heads > 1 && t.stride_head < dim))
        return Q2D_EINVAL;
    return Q2D_OK;
}

q2d_status check_sizes(const q2d_attention *a)
{
    if (!a) return Q2D_EINVAL;
    if (a->dtype != Q2D_F32 && a->dtype != Q2D_BF16) return Q2D_EINVAL;
    if ((a->causal != 0 && a->causal != 1) || a->batch <= 0 || a->heads_q <= 0 || a->heads_kv <= 0 || a->dim <= 0 ||
        a->len_q <= 0 || a->len_k <= 0 || a->window < 0)
        return Q2D_EINVAL;
    if (a->heads_q % a->heads_kv != 0) return Q2D_EINVAL;
    if (!(a->scale > 0.f) || !isfinite(a->scale) || !(a->softcap >= 0.f) || !isfinite(a->softcap)) return Q2D_EINVAL;
    if (a->dim % 8 != 0 || a->dim > 128 || a->len_q > kMaxLen || a->len_k > kMaxLen) return Q2D_EUNSUPPORTED;
    int64_t rows, n;
    if (__builtin_mul_overflow((int64_t)a->batch * a->heads_q, a->len_q > a->len_k ? a->len_q : a->len_k, &rows) ||
        __builtin_mul_overflow(rows, (int64_t)1024, &n))
        return Q2D_EUNSUPPORTED;
    return Q2D_OK;
}

q2d_status check(const q2d_attention *a)
{
    q2d_status s = check_sizes(a);
    if (s != Q2D_OK) return s;
    const int per = a->dtype == Q2D_F32 ? 4 : 8;
    s = check_heads(a->q, a->batch, a->len_q, a->heads_q, a->dim, per);
    if (s == Q2D_OK) s = check_heads(a->k, a->batch, a->len_k, a->heads_kv, a->dim, per);
    if (s == Q2D_OK) s = check_heads(a->v, a->batch, a->len_k, a->heads_kv, a->dim, per);
    if (s == Q2D_OK) s = check_output(a->out, a->batch, a->len_q, a->heads_q, a->dim, per);
    if (s != Q2D_OK) return s;
    auto word = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; };
    if (!word(a->slopes) || !word(a->documents) || !word(a->prefix) || !word(a->lse)) return Q2D_EINVAL;
    return Q2D_OK;
}

HeadsView view(const q2d_heads &t) { return {t.data, t.stride_batch, t.stride_length, t.stride_head}; }

int64_t ranges_bytes(const q2d_attention *a)
{
    return a->documents ? up256((int64_t)a->batch * ((a->len_k + 63) / 64) * 8) : 0;
}

int64_t workspace_of(const q2d_attention *a, bool backward)
{
    return ranges_bytes(a) + (backward ? up256((int64_t)a->batch * a->heads_q * a->len_q * 4) : 0);
}

AttentionArgs make_args(const q2d_attention *a, void *workspace)
{
    AttentionArgs r = {};
    r.q = view(a->q); r.k = view(a->k); r.v = view(a->v); r.out = view(a->out);
    r.lse = a->lse;
    r.ranges = reinterpret_cast<int2 *>(workspace);
    r.delta = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(workspace) + ranges_bytes(a));
    r.mask.causal = a->causal;
    // (no distance reaches 2^30)
    r.mask.window = (int32_t)(a->window > kMaxLen ? kMaxLen : a->window);
    r.mask.scale = a->scale; r.mask.cap = a->softcap;
    r.mask.slopes = a->slopes; r.mask.documents = a->documents; r.mask.prefix = a->prefix;
    r.batch = a->batch; r.len_q = (int32_t)a->len_q; r.len_k = (int32_t)a->len_k;
    r.heads_q = a->heads_q; r.heads_kv = a->heads_kv; r.dim = a->dim;
    return r;
}

q2d_status check_workspace(int64_t need, const void *workspace, int64_t bytes)
{
    if (need == 0) return Q2D_OK;
    if (!workspace || bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return Q2D_EINVAL;
    return Q2D_OK;
}

}  // namespace

extern "C" {

int64_t q2d_attention_workspace(const q2d_attention *a, int backward)
{
    if (check_sizes(a) != Q2D_OK || (backward != 0 && backward != 1)) return -1;
    return workspace_of(a, backward != 0);
}

q2d_status q2d_attention_fwd(const q2d_attention *a, void *workspace, int64_t workspace_bytes, hipStream_t stream)
{
    q2d_status s = check(a);
    if (s == Q2D_OK) s = check_workspace(workspace_of(a, false), workspace, workspace_bytes);
    if (s != Q2D_OK) return s;
    if (launch_attention_fwd(make_args(a, workspace), a->dtype == Q2D_F32, stream) != hipSuccess) return Q2D_ELAUNCH;
    return Q2D_OK;
}

q2d_status q2d_attention_bwd(const q2d_attention *a, const q2d_heads *dout, const q2d_heads *dq, const q2d_heads *dk,
                             const q2d_heads *dv, void *workspace, int64_t workspace_bytes, hipStream_t stream)
{
    q2d_status s = check(a);
    if (s != Q2D_OK) return s;
    if (!a->lse || !dout || !dq || !dk || !dv) return Q2D_EINVAL;
    const int per = a->dtype == Q2D_F32 ? 4 : 8;
    s = check_heads(*dout, a->batch, a->len_q, a->heads_q, a->dim, per);
    if (s == Q2D_OK) s = check_output(*dq, a->batch, a->len_q, a->heads_q, a->dim, per);
    if (s == Q2D_OK) s = check_output(*dk, a->batch, a->len_k, a->heads_kv, a->dim, per);
    if (s == Q2D_OK) s = check_output(*dv, a->batch, a->len_k, a->heads_kv, a->dim, per);
    if (s == Q2D_OK) s = check_workspace(workspace_of(a, true), workspace, workspace_bytes);
    if (s != Q2D_OK) return s;
    AttentionArgs r = make_args(a, workspace);
    r.dout = view(*dout); r.dq = view(*dq); r.dk = view(*dk); r.dv = view(*dv);
    if (launch_attention_bwd(r, a->dtype == Q2D_F32, stream) != hipSuccess) return Q2D_ELAUNCH;
    return Q2D_OK;
}

}  // extern "C"
