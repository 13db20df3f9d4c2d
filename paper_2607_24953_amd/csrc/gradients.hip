// 2-norm over many tensors, and their scaling.
//
// A launch takes up to kTensors tensors as kernel arguments, so that no table has to be copied to
// the device.  They are cut into pieces of kPiece elements; a workgroup takes every gridDim.x-th
// piece and writes one partial sum, in 64 bits: squares of float32 neither overflow nor vanish
// there, and the order of the additions is fixed.  The scaling kernel's workgroups each add all
// partial sums up again, in the same order, which saves a launch between the two.
#include "q2d.h"
#include "kernels.hpp"
#include "layout.hpp"
#include "norm_common.hpp"

#include <algorithm>
#include <math.h>
#include <new>
#include <vector>

namespace q2d {

namespace {

constexpr int kTensors = 128;
constexpr int64_t kPiece = 16384;
constexpr int kMaxParts = 2048;

struct Tensors {
    const void *data[kTensors];
    void *out[kTensors];
    int64_t count[kTensors];
    int32_t first[kTensors];       // the tensor's first piece
    int32_t n, pieces;
    uint32_t bf16[kTensors / 32];  // a bit a tensor
};

// tensor of a piece
__device__ __forceinline__ int tensor_of(const Tensors &t, int piece) { return seg_search(t.first, t.n, piece); }

__device__ __forceinline__ bool is_bf16(const Tensors &t, int i) { return (t.bf16[i >> 5] >> (i & 31)) & 1; }

// Eight-element chunks that a lane has in flight, and of a piece
constexpr int kFlight = 4, kChunks = (int)(kPiece / (8 * 256));

template <bool BF16>
__device__ __forceinline__ double square_piece(const void *data, int64_t at, int64_t left)
{
    const uint8_t *p = reinterpret_cast<const uint8_t *>(data) + at * (BF16 ? 2 : 4);
    double s = 0.0;
#pragma unroll 1
    for (int k0 = 0; k0 < kChunks; k0 += kFlight) {
        Eight<BF16> e[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const int c = 8 * ((k0 + k) * 256 + threadIdx.x);
            e[k].load(p + c * (BF16 ? 2 : 4), left - c);
        }
#pragma unroll
        for (int k = 0; k < kFlight; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double v = e[k].at(j);
                s = __builtin_fma(v, v, s);
            }
    }
    return s;
}

__global__ __launch_bounds__(256) void grad_square_kernel(const Tensors t, double *parts)
{
    __shared__ double lds[4];
    double s = 0.0;
    for (int piece = blockIdx.x; piece < t.pieces; piece += gridDim.x) {
        const int i = tensor_of(t, piece);
        const int64_t at = (piece - t.first[i]) * kPiece, left = t.count[i] - at;
        s += is_bf16(t, i) ? square_piece<true>(t.data[i], at, left) : square_piece<false>(t.data[i], at, left);
    }
    s = group_sum(s, 4, lds);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// square root of the sum of all parts, the same value in every lane
__device__ __forceinline__ double total_norm(const double *parts, int n, double *lds)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) s += parts[i];
    return __builtin_sqrt(group_sum(s, 4, lds));
}

__global__ __launch_bounds__(256) void grad_norm_kernel(const double *parts, int n, float *norm)
{
    __shared__ double lds[4];
    const double s = total_norm(parts, n, lds);
    if (threadIdx.x == 0) *norm = (float)s;
}

template <bool BF16>
__device__ __forceinline__ void scale_piece(const void *data, void *out, int64_t at, int64_t left, bool clip, float f)
{
    const uint8_t *p = reinterpret_cast<const uint8_t *>(data) + at * (BF16 ? 2 : 4);
    uint8_t *o = reinterpret_cast<uint8_t *>(out) + at * (BF16 ? 2 : 4);
#pragma unroll 1
    for (int k0 = 0; k0 < kChunks; k0 += kFlight) {
        Eight<BF16> e[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const int c = 8 * ((k0 + k) * 256 + threadIdx.x);
            e[k].load(p + c * (BF16 ? 2 : 4), left - c);
        }
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const int c = 8 * ((k0 + k) * 256 + threadIdx.x);
            if (clip) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = e[k].at(j) * f;
                e[k].set(v);
            }
            e[k].store(o + c * (BF16 ? 2 : 4), left - c);
        }
    }
}

// (the last pieces first: the square sums read them last, and some are still in the cache)
__global__ __launch_bounds__(256) void grad_scale_kernel(const Tensors t, const double *parts, int n, const float *given,
                                                         double max_norm, float *norm)
{
    __shared__ double lds[4];
    const double total = parts ? total_norm(parts, n, lds) : (double)*given;
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    // a norm that is not finite leaves the gradients as they are
    const bool clip = (float)total < __builtin_inff() && total > max_norm;
    const float f = clip ? (float)(max_norm / total) : 1.f;
    for (int piece = t.pieces - 1 - (int)blockIdx.x; piece >= 0; piece -= gridDim.x) {
        const int i = tensor_of(t, piece);
        if (!clip && t.out[i] == t.data[i]) continue;
        const int64_t at = (piece - t.first[i]) * kPiece, left = t.count[i] - at;
        if (is_bf16(t, i)) scale_piece<true>(t.data[i], t.out[i], at, left, clip, f);
        else scale_piece<false>(t.data[i], t.out[i], at, left, clip, f);
    }
}

struct Set {
    int32_t n;
    const void *const *data;
    void *const *out;
    const int64_t *counts;
    const int32_t *dtypes;
};

q2d_status check_set(const Set &g)
{
    if (g.n < 0 || (g.n > 0 && (!g.data || !g.counts || !g.dtypes))) return Q2D_EINVAL;
    int64_t pieces = 0;
    for (int32_t i = 0; i < g.n; ++i) {
        if (!valid_dtype((q2d_dtype)g.dtypes[i]) || g.counts[i] < 0) return Q2D_EINVAL;
        if (g.counts[i] > int64_t(1) << 40) return Q2D_EUNSUPPORTED;
        if (g.counts[i] == 0) continue;
        const uintptr_t size = (uintptr_t)dtype_bytes((q2d_dtype)g.dtypes[i]);
        if (!g.data[i] || !aligned(g.data[i], size)) return Q2D_EINVAL;
        if (g.out && (!g.out[i] || !aligned(g.out[i], size))) return Q2D_EINVAL;
        pieces += cdiv(g.counts[i], kPiece);
        if (pieces > INT32_MAX) return Q2D_EUNSUPPORTED;
    }
    return Q2D_OK;
}

// Whether what the call writes meets anything else that it reads or writes: an output may be its
// own input, in place, and nothing else.
q2d_status check_apart(const Set &g)
{
    struct Range { uintptr_t at, end; int32_t i; bool out; };
    std::vector<Range> r;
    try {
        r.reserve(2 * (size_t)g.n);
        for (int32_t i = 0; i < g.n; ++i) {
            const uintptr_t bytes = (uintptr_t)g.counts[i] * dtype_bytes((q2d_dtype)g.dtypes[i]);
            if (!bytes) continue;
            const uintptr_t d = reinterpret_cast<uintptr_t>(g.data[i]), o = g.out ? reinterpret_cast<uintptr_t>(g.out[i]) : d;
            r.push_back({o, o + bytes, i, true});
            if (o != d) r.push_back({d, d + bytes, i, false});
        }
    } catch (const std::bad_alloc &) {
        return Q2D_EUNSUPPORTED;
    }
    std::sort(r.begin(), r.end(), [](const Range &a, const Range &b) { return a.at < b.at; });
    // the furthest ends so far, of outputs and of all: inputs may share memory with one another
    uintptr_t end_out = 0, end_all = 0;
    for (const Range &x : r) {
        if (x.at < end_out || (x.out && x.at < end_all)) return Q2D_EINVAL;
        if (x.out) end_out = std::max(end_out, x.end);
        end_all = std::max(end_all, x.end);
    }
    return Q2D_OK;
}

int64_t launches_of(int32_t n) { return (n + kTensors - 1) / kTensors; }

// Partial sums of a call at most: kMaxParts shared by its launches, one a launch at least
int64_t parts_of(int32_t n) { return kMaxParts + launches_of(n); }

// Runs f(tensors, workgroups) for each launch of a set; false for an error of the runtime
template <typename F>
bool for_launches(const Set &g, F f)
{
    int64_t all = 0;
    for (int32_t i = 0; i < g.n; ++i) all += cdiv(g.counts[i], kPiece);
    for (int32_t i = 0; i < g.n;) {
        Tensors t;
        t.n = 0;
        int64_t pieces = 0;
        for (auto &b : t.bf16) b = 0;
        for (; i < g.n && t.n < kTensors; ++i) {
            if (g.counts[i] == 0) continue;
            t.data[t.n] = g.data[i];
            t.out[t.n] = g.out ? g.out[i] : const_cast<void *>(g.data[i]);
            t.count[t.n] = g.counts[i];
            t.first[t.n] = (int32_t)pieces;
            if (g.dtypes[i] == Q2D_BF16) t.bf16[t.n >> 5] |= 1u << (t.n & 31);
            pieces += cdiv(g.counts[i], kPiece);
            ++t.n;
        }
        if (t.n == 0) break;
        t.pieces = (int32_t)pieces;
        for (int k = t.n; k < kTensors; ++k) {
            t.data[k] = nullptr; t.out[k] = nullptr; t.count[k] = 0; t.first[k] = t.pieces;
        }
        if (!f(t, (unsigned)std::min<int64_t>(pieces, std::max<int64_t>(1, kMaxParts * pieces / all)))) return false;
    }
    return true;
}

// Partial sums of the set into parts; their number, or -1
int square_sums(const Set &g, double *parts, hipStream_t stream)
{
    int n = 0;
    const bool ok = for_launches(g, [&](const Tensors &t, unsigned groups) {
        hipLaunchKernelGGL(grad_square_kernel, dim3(groups), dim3(256), 0, stream, t, parts + n);
        n += (int)groups;
        return hipGetLastError() == hipSuccess;
    });
    return ok ? n : -1;
}

}  // namespace

}  // namespace q2d

using namespace q2d;

extern "C" {

int64_t q2d_grad_workspace(int32_t n) { return n < 0 ? -1 : parts_of(n) * (int64_t)sizeof(double); }

q2d_status q2d_grad_norm(int32_t n, const void *const *data, const int64_t *counts, const int32_t *dtypes, float *norm,
                         void *workspace, int64_t workspace_bytes, hipStream_t stream)
{
    const Set g = {n, data, nullptr, counts, dtypes};
    const q2d_status s = check_set(g);
    if (s != Q2D_OK) return s;
    if (!norm || !aligned(norm, 4) || !workspace || !aligned(workspace, 8) || workspace_bytes < q2d_grad_workspace(n)) return Q2D_EINVAL;
    double *parts = reinterpret_cast<double *>(workspace);
    const int k = square_sums(g, parts, stream);
    if (k < 0) return Q2D_ELAUNCH;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, stream, parts, k, norm);
    return hipGetLastError() == hipSuccess ? Q2D_OK : Q2D_ELAUNCH;
}

q2d_status q2d_clip_grads(int32_t n, const void *const *data, void *const *out, const int64_t *counts, const int32_t *dtypes,
                          double max_norm, const float *given, float *norm, void *workspace, int64_t workspace_bytes,
                          hipStream_t stream)
{
    const Set g = {n, data, out, counts, dtypes};
    q2d_status s = check_set(g);
    if (s == Q2D_OK) s = check_apart(g);
    if (s != Q2D_OK) return s;
    if (!(max_norm >= 0.0) || !std::isfinite(max_norm)) return Q2D_EINVAL;
    // either a norm to go by, or a place for the norm
    const float *one = given ? given : norm;
    if (!one || (given && norm) || !aligned(one, 4)) return Q2D_EINVAL;
    double *parts = nullptr;
    int k = 0;
    if (!given) {
        if (!workspace || !aligned(workspace, 8) || workspace_bytes < q2d_grad_workspace(n)) return Q2D_EINVAL;
        parts = reinterpret_cast<double *>(workspace);
        k = square_sums(g, parts, stream);
        if (k < 0) return Q2D_ELAUNCH;
        if (k == 0) {       // no elements: nothing to scale
            hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, stream, parts, 0, norm);
            return hipGetLastError() == hipSuccess ? Q2D_OK : Q2D_ELAUNCH;
        }
    }
    const bool ok = for_launches(g, [&](const Tensors &t, unsigned groups) {
        hipLaunchKernelGGL(grad_scale_kernel, dim3(groups), dim3(256), 0, stream, t, parts, k, given, max_norm, norm);
        norm = nullptr;      // (written by the first launch)
        return hipGetLastError() == hipSuccess;
    });
    return ok ? Q2D_OK : Q2D_ELAUNCH;
}

}  // extern "C"
