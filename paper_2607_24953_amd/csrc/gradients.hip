// 2-norm over many tensors, and their scaling.
//
// A launch takes its tensors as kernel arguments, as many as fit 4 KB, so that no table has to be
// copied to the device.  They are cut into pieces of one size, the last of a tensor shorter; a
// workgroup takes every gridDim.x-th piece and writes one partial sum, in 64 bits: squares of float32
// neither overflow nor vanish there, and the order of the additions is fixed.  The scaling
// kernel's workgroups each add all partial sums up again, in the same order, which saves a
// launch between the two.
//
// The memory bounds both: 405M float32 are read in 259 us (6.3 TB/s) and scaled in 584 (5.5 TB/s); 98M
// bfloat16 of 240 tensors in 39 and 46 + 27.  With 128 tensors a launch the latter took 58 + 82 us.
#include "q2d.h"
#include "kernels.hpp"
#include "layout.hpp"
#include "norm_common.hpp"

#include <algorithm>
#include <exception>
#include <math.h>
#include <vector>

namespace q2d {

namespace {

// elements of a turn of a workgroup's 256 lanes, eight each; a piece is 1 to kTurns of them
constexpr int kTurn = 2048, kTurns = 8;
constexpr int kMaxParts = 2048;

// N tensors; SCALED: with a place for the results
template <int N, bool SCALED>
struct Tensors {
    const void *data[N];
    void *out[SCALED ? N : 1];
    int32_t first[N];              // a tensor's first piece
    int32_t last[N];               // elements of its last one
    int32_t n, pieces, turns;
    uint32_t bf16[(N + 31) / 32];  // a bit a tensor
    static constexpr int kMost = N;
    static constexpr bool kScaled = SCALED;
};
typedef Tensors<240, false> Squared;
typedef Tensors<160, true> Scaled;
static_assert(sizeof(Squared) + 8 <= 4096 && sizeof(Scaled) + 40 <= 4096, "kernel arguments");

// A piece: its tensor, first element and length
struct Piece { int tensor; bool bf16; int64_t at; int length; };
template <typename T>
__device__ __forceinline__ Piece piece_of(const T &t, int piece)
{
    const int i = seg_search(t.first, t.n, piece), size = t.turns * kTurn;
    const bool last = piece + 1 == (i + 1 < t.n ? t.first[i + 1] : t.pieces);
    return {i, (bool)((t.bf16[i >> 5] >> (i & 31)) & 1), (int64_t)(piece - t.first[i]) * size, last ? t.last[i] : size};
}

// 16 bytes of a tensor.  (With eight float32 a lane each of its two loads took every other 16 bytes
// of its lines: 150M float32 clipped 337 us, so 306)
template <bool BF16>
struct Unit : Run<BF16, BF16 ? 8 : 4> {
    static constexpr int kN = BF16 ? 8 : 4, kBytes = 16 / kN;
    __device__ __forceinline__ void scale(float f)
    {
        float v[kN];
#pragma unroll
        for (int j = 0; j < kN; ++j) v[j] = this->at(j) * f;
        this->set(v);
    }
};

// 16-byte accesses that a lane has in flight
template <bool BF16> constexpr int kFlight = BF16 ? 4 : 2;

// (ONCE: no second pass follows)
template <bool BF16, bool ONCE>
__device__ __forceinline__ double square_piece(const void *data, int64_t at, int length)
{
    typedef Unit<BF16> U;
    constexpr int kUnits = kFlight<BF16>, kStep = 256 * U::kN;
    const uint8_t *p = reinterpret_cast<const uint8_t *>(data) + at * U::kBytes;
    double s = 0.0;
#pragma unroll 1
    for (int c0 = U::kN * threadIdx.x; c0 < length; c0 += kUnits * kStep) {
        U e[kUnits];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int c = c0 + k * kStep;
            e[k].template load<ONCE>(p + c * U::kBytes, length - c);
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k)
#pragma unroll
            for (int j = 0; j < U::kN; ++j) {
                const double v = e[k].at(j);
                s = __builtin_fma(v, v, s);
            }
    }
    return s;
}

template <bool ONCE>
__global__ __launch_bounds__(256) void grad_square_kernel(const Squared t, double *parts)
{
    __shared__ double lds[4];
    double s = 0.0;
    for (int piece = blockIdx.x; piece < t.pieces; piece += gridDim.x) {
        const Piece p = piece_of(t, piece);
        s += p.bf16 ? square_piece<true, ONCE>(t.data[p.tensor], p.at, p.length) : square_piece<false, ONCE>(t.data[p.tensor], p.at, p.length);
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
__device__ __forceinline__ void scale_piece(const void *data, void *out, int64_t at, int length, bool clip, float f)
{
    typedef Unit<BF16> U;
    constexpr int kUnits = kFlight<BF16>, kStep = 256 * U::kN;
    const uint8_t *p = reinterpret_cast<const uint8_t *>(data) + at * U::kBytes;
    uint8_t *o = reinterpret_cast<uint8_t *>(out) + at * U::kBytes;
#pragma unroll 1
    for (int c0 = U::kN * threadIdx.x; c0 < length; c0 += kUnits * kStep) {
        U e[kUnits];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int c = c0 + k * kStep;
            e[k].template load<true>(p + c * U::kBytes, length - c);
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int c = c0 + k * kStep;
            if (clip) e[k].scale(f);
            e[k].template store<true>(o + c * U::kBytes, length - c);
        }
    }
}

// The last pieces first, past the cache: the square sums read them last, and what the cache still
// holds of them is not pushed out by what is written here (98M bfloat16 124 us, so 99; 400M
// 845 -> 821)
__global__ __launch_bounds__(256) void grad_scale_kernel(const Scaled t, const double *parts, int n, const float *given,
                                                         double max_norm, float *norm)
{
    __shared__ double lds[4];
    const double total = parts ? total_norm(parts, n, lds) : (double)*given;
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    // a norm that is not finite leaves the gradients as they are
    const bool clip = (float)total < __builtin_inff() && total > max_norm;
    const float f = clip ? (float)(max_norm / total) : 1.f;
    for (int piece = t.pieces - 1 - (int)blockIdx.x; piece >= 0; piece -= gridDim.x) {
        const Piece p = piece_of(t, piece);
        if (!clip && t.out[p.tensor] == t.data[p.tensor]) continue;
        if (p.bf16) scale_piece<true>(t.data[p.tensor], t.out[p.tensor], p.at, p.length, clip, f);
        else scale_piece<false>(t.data[p.tensor], t.out[p.tensor], p.at, p.length, clip, f);
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
        pieces += cdiv(g.counts[i], kTurn);
        if (pieces > INT32_MAX) return Q2D_EUNSUPPORTED;
    }
    return Q2D_OK;
}

// Whether what the call writes meets anything else that it reads or writes: a tensor's output may be
// its own input, in place, and nothing else.  given, norm and the workspace: where not null.
q2d_status check_apart(const Set &g, const void *given, const void *norm, const void *workspace, int64_t workspace_bytes)
{
    struct Range { uintptr_t at, end; bool out; };
    std::vector<Range> r;
    auto add = [&](const void *p, uintptr_t bytes, bool out) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p && bytes) r.push_back({at, at + bytes, out});
    };
    try {
        r.reserve(2 * (size_t)g.n + 3);
        for (int32_t i = 0; i < g.n; ++i) {
            const uintptr_t bytes = (uintptr_t)g.counts[i] * dtype_bytes((q2d_dtype)g.dtypes[i]);
            const void *out = g.out ? g.out[i] : g.data[i];
            add(out, bytes, true);
            if (out != g.data[i]) add(g.data[i], bytes, false);
        }
        add(given, 4, false);
        add(norm, 4, true);
        add(workspace, (uintptr_t)workspace_bytes, true);
        std::sort(r.begin(), r.end(), [](const Range &a, const Range &b) { return a.at < b.at; });
    } catch (const std::exception &) {
        return Q2D_EUNSUPPORTED;
    }
    // the furthest ends so far, of outputs and of all: inputs may share memory with one another
    uintptr_t end_out = 0, end_all = 0;
    for (const Range &x : r) {
        if (x.at < end_out || (x.out && x.at < end_all)) return Q2D_EINVAL;
        if (x.out) end_out = std::max(end_out, x.end);
        end_all = std::max(end_all, x.end);
    }
    return Q2D_OK;
}

// The same for q2d_grad_norm, where the tensors are read only
bool norm_apart(const Set &g, const void *norm, const void *workspace, int64_t workspace_bytes)
{
    const uintptr_t n = reinterpret_cast<uintptr_t>(norm), w = reinterpret_cast<uintptr_t>(workspace), w_end = w + (uintptr_t)workspace_bytes;
    bool apart = n >= w_end || n + 4 <= w;
    for (int32_t i = 0; i < g.n; ++i) {
        if (g.counts[i] == 0) continue;
        const uintptr_t at = reinterpret_cast<uintptr_t>(g.data[i]), end = at + (uintptr_t)g.counts[i] * dtype_bytes((q2d_dtype)g.dtypes[i]);
        apart &= (n >= end || n + 4 <= at) && (w >= end || w_end <= at);
    }
    return apart;
}

// Partial sums of a call at most: kMaxParts shared by its launches, one a launch at least
int64_t parts_of(int32_t n) { return kMaxParts + n / Squared::kMost + 1; }

// Fills t with the tensors of a set from i on, as many as fit; the first one that did not
template <typename T>
int32_t fill(const Set &g, int32_t i, int turns, T &t)
{
    const int64_t size = turns * (int64_t)kTurn;
    int64_t pieces = 0;
    t = T{};
    for (; i < g.n && t.n < T::kMost; ++i) {
        if (g.counts[i] == 0) continue;
        const int64_t k = cdiv(g.counts[i], size);
        t.data[t.n] = g.data[i];
        if (T::kScaled) t.out[t.n] = g.out ? g.out[i] : const_cast<void *>(g.data[i]);
        t.first[t.n] = (int32_t)pieces;
        t.last[t.n] = (int32_t)(g.counts[i] - (k - 1) * size);
        if (g.dtypes[i] == Q2D_BF16) t.bf16[t.n >> 5] |= 1u << (t.n & 31);
        pieces += k;
        ++t.n;
    }
    t.pieces = (int32_t)pieces;
    t.turns = turns;
    return i;
}

int64_t elements(const Set &g)
{
    int64_t all = 0;
    for (int32_t i = 0; i < g.n; ++i) all += g.counts[i];
    return all;
}

// Turns of a piece: a workgroup for each of 1024 pieces first, then longer ones.  (In one size of
// 8 turns the 0.8 M float32 of a small model's gradients took 5.1 us for their squares.)
int turns_of(int64_t all)
{
    int t = 1;
    while (t < kTurns && all / (2 * t * kTurn) >= 1024) t *= 2;
    return t;
}

// Partial sums of the set into parts; their number, or -1
int square_sums(const Set &g, int64_t all, bool once, double *parts, hipStream_t stream)
{
    const int turns = turns_of(all);
    int64_t pieces = 0;
    for (int32_t i = 0; i < g.n; ++i) pieces += cdiv(g.counts[i], turns * (int64_t)kTurn);
    int n = 0;
    Squared t;
    for (int32_t i = 0; i < g.n;) {
        i = fill(g, i, turns, t);
        if (t.n == 0) break;
        // a launch's share of kMaxParts, by its pieces: all shares, each rounded down, stay within it
        const int groups = (int)std::min<int64_t>(t.pieces, std::max<int64_t>(1, kMaxParts * (int64_t)t.pieces / pieces));
        if (once) hipLaunchKernelGGL(grad_square_kernel<true>, dim3(groups), dim3(256), 0, stream, t, parts + n);
        else hipLaunchKernelGGL(grad_square_kernel<false>, dim3(groups), dim3(256), 0, stream, t, parts + n);
        if (hipGetLastError() != hipSuccess) return -1;
        n += groups;
    }
    return n;
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
    if (!norm_apart(g, norm, workspace, q2d_grad_workspace(n))) return Q2D_EINVAL;
    double *parts = reinterpret_cast<double *>(workspace);
    const int k = square_sums(g, elements(g), true, parts, stream);
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
    if (s != Q2D_OK) return s;
    if (!(max_norm >= 0.0) || !std::isfinite(max_norm)) return Q2D_EINVAL;
    // either a norm to go by, or a place for the norm
    const float *one = given ? given : norm;
    if (!one || (given && norm) || !aligned(one, 4)) return Q2D_EINVAL;
    if (!given && (!workspace || !aligned(workspace, 8) || workspace_bytes < q2d_grad_workspace(n))) return Q2D_EINVAL;
    s = check_apart(g, given, norm, given ? nullptr : workspace, q2d_grad_workspace(n));
    if (s != Q2D_OK) return s;
    double *parts = nullptr;
    int k = 0;
    const int64_t all = elements(g);
    if (!given) {
        parts = reinterpret_cast<double *>(workspace);
        k = square_sums(g, all, false, parts, stream);
        if (k < 0) return Q2D_ELAUNCH;
        if (k == 0) {       // no elements: nothing to scale
            hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, stream, parts, 0, norm);
            return hipGetLastError() == hipSuccess ? Q2D_OK : Q2D_ELAUNCH;
        }
    }
    const int turns = turns_of(all);
    Scaled t;
    for (int32_t i = 0; i < n;) {
        i = fill(g, i, turns, t);
        if (t.n == 0) break;
        const dim3 groups(std::min(t.pieces, kMaxParts));
        hipLaunchKernelGGL(grad_scale_kernel, groups, dim3(256), 0, stream, t, parts, k, given, max_norm, norm);
        if (hipGetLastError() != hipSuccess) return Q2D_ELAUNCH;
        norm = nullptr;     // (written by the first launch)
    }
    return Q2D_OK;
}

}  // extern "C"
