// Attention of new tokens over the paged 8-bit cache.
//
// The query rows that share a key head (group heads x new tokens) are the columns of 16-wide
// tiles; a wave walks super-blocks of 64 tokens and takes codes straight from memory into
// MFMA operands: 16 bytes a lane along a key's dims, and along tokens of the transposed
// values, converted exactly to bfloat16 (v_cvt_scalef32_pk_bf16_fp8).  No LDS and no
// exchange between lanes stands between the cache and the products:
//   S^T = K Q^T as 16 x 16 tiles u = 0..3 whose row 4 g + i is token 16 g + 4 u + i, so that
//   lane group g = lane / 16 ends with tokens 16 g .. 16 g + 15 of its query column, which
//   is the order in which its 16-byte value loads hold them;  O^T += V^T P^T.
// Key scales multiply scores, value scales enter the conversion; both are one number a lane.
//
// With few query rows the time goes into reading the cache: a sequence's tokens are dealt to
// the waves of several workgroups, the waves of one join through LDS and the workgroups
// through a second kernel.
#include "attention_common.hpp"
#include "cache_common.hpp"

namespace q2d {

namespace {

constexpr int kSuper = 64;
constexpr uint32_t kNoBlock = 256;             // in place of a scale byte

__device__ __forceinline__ bf16x8 fp8_to_bf16(uint32_t lo, uint32_t hi, float scale)
{
    const bf16x2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    const bf16x2v b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    const bf16x2v d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// codes of one super-block in a lane: keys [tile u][64 dims], values [16 dims], scale bytes
template <int DT>
struct Codes {
    u4v k[4][DT / 64], v[DT / 16];
    uint32_t ks, vs;
};

// The cache blocks of super-block sb that this lane reads: of its key rows, and of its values
// and scores (-1: none)
struct Where {
    int64_t key, value;
};

__device__ __forceinline__ Where locate(const CachedArgs &a, int b, int head, int sb, int len, int lane)
{
    // key rows of lane: tokens 16 (r / 4) + .., r = lane % 16: block r / 8; values: block g / 2
    const int kb = 2 * sb + ((lane >> 3) & 1), vb = 2 * sb + (lane >> 5);
    Where w = {-1, -1};
    if (kb * kBlockTokens < len) w.key = cache_block(a.cache, a.seq, b, kb, head);
    if (vb * kBlockTokens < len) w.value = cache_block(a.cache, a.seq, b, vb, head);
    return w;
}

template <int DT>
__device__ __forceinline__ void fetch(const CachedArgs &a, const Where &w, int lane, Codes<DT> &c)
{
    const int D = a.cache.dim, r = lane & 15, g = lane >> 4;
    const u4v zero = {0, 0, 0, 0};
    const uint8_t *kp = a.cache.k + (w.key < 0 ? 0 : w.key) * kBlockTokens * D + (16 * ((r >> 2) & 1) + (r & 3)) * D;
    const uint8_t *vp = a.cache.v + (w.value < 0 ? 0 : w.value) * kBlockTokens * D + r * kBlockTokens + 16 * (g & 1);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int t = 0; t < DT / 64; ++t) {
            const int d = 64 * t + 16 * g;
            c.k[u][t] = w.key >= 0 && d < D ? *reinterpret_cast<const u4v *>(kp + 4 * u * D + d) : zero;
        }
#pragma unroll
    for (int t = 0; t < DT / 16; ++t)
        c.v[t] = w.value >= 0 && 16 * t < D ? *reinterpret_cast<const u4v *>(vp + 16 * t * kBlockTokens) : zero;
    c.ks = w.value >= 0 ? a.cache.ks[w.value] : 0u;
    c.vs = w.value >= 0 ? a.cache.vs[w.value] : kNoBlock;
}

// MODS bit 0: capped scores, bit 1: distance bias; NT: 16-column tiles of query rows
template <int DT, int MODS, int NT>
__global__ __launch_bounds__(256, 1) void attention_cached_kernel(const CachedArgs a)
{
    constexpr bool CAP = MODS & 1, BIAS = MODS & 2;
    constexpr int KS = DT / 32, VT = DT / 16, ROWS = 16 * NT;
    // two waves' sums [row][dim] at a time, and all waves' statistics
    __shared__ __align__(16) float osum[2][ROWS * DT];
    __shared__ float stat[2][4][ROWS];

    const AttentionMask &m = a.mask;
    const int group = a.heads_q / a.cache.heads, D = a.cache.dim;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int split = blockIdx.x % a.splits;
    const int64_t rest = blockIdx.x / a.splits;
    const int head = (int)(rest % a.cache.heads);
    const int64_t tile = rest / a.cache.heads;
    Span s;
    int rt;
    const int b = find_unit(a.seq, a.cache.page_blocks * kBlockTokens, tile,
                            [&](const Span &x) { return (int)(((int64_t)x.n * group + ROWS - 1) / ROWS); }, s, rt);
    if (b < 0) return;

    // this lane's query rows: column c of tile nt
    const int rows = min(ROWS, (int)((int64_t)s.n * group - (int64_t)rt * ROWS));
    const int nts = (rows + 15) / 16;
    int tok[NT], hq[NT], pos[NT];
    bool row[NT];
    bf16x8 qf[NT][KS];
    float slope[NT];
    ScoreMap sm = score_map(m, 0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int c = nt * 16 + col, r = rt * ROWS + c;
        row[nt] = c < rows;
        tok[nt] = r / group;
        hq[nt] = head * group + r % group;
        pos[nt] = s.len - s.n + tok[nt];
        const __bf16 *q = (const __bf16 *)a.q + (s.tok0 + tok[nt]) * a.q_st + hq[nt] * a.q_sh;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            // the order of dims in which a 16-byte load of codes serves two steps
            const int d = 64 * (ks >> 1) + 16 * g + 8 * (ks & 1);
            bf16x8 x = {};
            if (row[nt] && d < D) x = *reinterpret_cast<const bf16x8 *>(q + d);
            qf[nt][ks] = x;
        }
        slope[nt] = BIAS && row[nt] ? m.slopes[hq[nt]] * kLog2e / sm.c : 0.f;
    }
    const int prefix = m.prefix ? min(max(m.prefix[b], 0), s.len) : 0;
    const int p0 = s.len - s.n + rt * ROWS / group, p1 = s.len - s.n + (rt * ROWS + rows - 1) / group;
    // tokens that some row sees: [t0, t1), and this workgroup's super-blocks of them
    int t1 = max(min(p1 + 1, s.len), prefix), t0 = m.window && !prefix ? max(p0 - m.window + 1, 0) : 0;
    if (t1 < t0) t1 = t0;
    const int sb0 = t0 / kSuper, sbs = (t1 + kSuper - 1) / kSuper - sb0;
    const int from = sb0 + (int)((int64_t)sbs * split / a.splits), to = sb0 + (int)((int64_t)sbs * (split + 1) / a.splits);

    v4f o[VT][NT] = {};
    float mx[NT], sum[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) { mx[nt] = -INFINITY; sum[nt] = 0.f; }
    const float thr = 8.f / sm.c;

    Codes<DT> c;
    Where ahead = {-1, -1};
    int sb = from + wave;
    if (sb < to) fetch<DT>(a, locate(a, b, head, sb, s.len, lane), lane, c);
    if (sb + 4 < to) ahead = locate(a, b, head, sb + 4, s.len, lane);
    for (; sb < to; sb += 4) {
        Codes<DT> next;
        if (sb + 4 < to) fetch<DT>(a, ahead, lane, next);
        if (sb + 8 < to) ahead = locate(a, b, head, sb + 8, s.len, lane);

        const int j0 = sb * kSuper;
        // values past the end: codes of 0 in place of what a page holds there
        if (j0 + kSuper > s.len) {
            const int n = min(max(s.len - (j0 + 16 * g), 0), 16);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int k = min(max(n - 4 * w, 0), 4);
                const uint32_t keep = k == 4 ? ~0u : (1u << (8 * k)) - 1;
#pragma unroll
                for (int t = 0; t < VT; ++t) c.v[t][w] &= keep;
            }
        }
        const float ks = c.ks == 255 ? __builtin_nanf("") : ldexpf(CAP ? sm.k1 : 1.f, (int)c.ks - 127);
        const bool all = j0 + kSuper - 1 <= p0 && j0 + kSuper <= s.len && (!m.window || p1 - j0 < m.window) &&
                         !__any(c.vs == kNoBlock);
        bf16x8 pf[NT][2];
        // (a value scale of 255 marks a block with a NaN: rows that see it get one)
        const bool bad = __any(c.vs == 255);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt >= nts) continue;
            v4f z[4] = {};
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int t = 0; t < DT / 64; ++t) {
                    const u4v w = c.k[u][t];
                    z[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_to_bf16(w[0], w[1], 1.f), qf[nt][2 * t], z[u], 0, 0, 0);
                    z[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_to_bf16(w[2], w[3], 1.f), qf[nt][2 * t + 1], z[u], 0, 0, 0);
                }
            const int jl = j0 + 16 * g;
            const float d0 = (float)(pos[nt] - jl);
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = z[u][i] * ks;
                    if constexpr (CAP) x = tanh_of(x, false);
                    if constexpr (BIAS) x = fmaf(-slope[nt], fabsf(d0 - (float)(4 * u + i)), x);
                    z[u][i] = x;
                }
            if (!all) {
                const Sight sight = query_sight(m, pos[nt], s.len, prefix, 0);
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = jl + 4 * u + i;
                        const bool ok = ((j >= sight.lo && j < sight.hi) || j < prefix) && c.vs != kNoBlock;
                        z[u][i] = ok ? z[u][i] : -INFINITY;
                    }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, z[u][i]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            // (as in the forward kernel: the maximum moves only where it is passed by 2^8)
            if (__any(top > mx[nt] + thr)) {
                const float now = fmaxf(mx[nt], top);
                const float f = mx[nt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mx[nt] - now) * sm.c);
#pragma unroll
                for (int t = 0; t < VT; ++t) o[t][nt] *= f;
                sum[nt] *= f;
                mx[nt] = now;
            }
            const float off = mx[nt] == -INFINITY ? 0.f : -mx[nt] * sm.c;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(z[u][i], sm.c, off));
                    sum[nt] += e;
                    z[u][i] = e;
                    if (bad && c.vs == 255 && e != 0.f) z[u][i] = __builtin_nanf("");
                }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) pf[nt][k][i] = (__bf16)z[2 * k + (i >> 2)][i & 3];
        }
        const float vs = bits_f((c.vs >= 255 ? 127u : c.vs) << 23);
#pragma unroll
        for (int t = 0; t < VT; ++t)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const bf16x8 x = fp8_to_bf16(c.v[t][2 * k], c.v[t][2 * k + 1], vs);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    if (nt < nts) o[t][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, pf[nt][k], o[t][nt], 0, 0, 0);
            }
        c = next;
    }

    // join the four waves: common maximum, then the sums in two steps
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        sum[nt] += __shfl_xor(sum[nt], 16);
        sum[nt] += __shfl_xor(sum[nt], 32);
        if (g == 0) {
            stat[0][wave][nt * 16 + col] = mx[nt];
            stat[1][wave][nt * 16 + col] = sum[nt];
        }
    }
    __syncthreads();
    float total[NT], most[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = nt * 16 + col;
        most[nt] = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) most[nt] = fmaxf(most[nt], stat[0][w][r]);
        total[nt] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            // (sums of nothing are 0; one that is NaN stays)
            const float x = stat[1][w][r], y = stat[0][w][r];
            total[nt] += x == 0.f ? 0.f : x * (y == most[nt] ? 1.f : __builtin_amdgcn_exp2f((y - most[nt]) * sm.c));
        }
        const float f = sum[nt] == 0.f ? 0.f : mx[nt] == most[nt] ? 1.f : __builtin_amdgcn_exp2f((mx[nt] - most[nt]) * sm.c);
#pragma unroll
        for (int t = 0; t < VT; ++t) o[t][nt] *= f;
    }
    auto put = [&](float *dst) {
#pragma unroll
        for (int t = 0; t < VT; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                *reinterpret_cast<v4f *>(dst + (nt * 16 + col) * DT + 16 * t + 4 * g) = o[t][nt];
    };
    auto add = [&](const float *src) {
#pragma unroll
        for (int t = 0; t < VT; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                o[t][nt] += *reinterpret_cast<const v4f *>(src + (nt * 16 + col) * DT + 16 * t + 4 * g);
    };
    if (wave >= 2) put(osum[wave - 2]);
    __syncthreads();
    if (wave < 2) add(osum[wave]);
    __syncthreads();
    if (wave == 1) put(osum[0]);
    __syncthreads();
    if (wave != 0) return;
    add(osum[0]);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        if (!row[nt]) continue;
        if (a.splits == 1) {
            const float inv = total[nt] == 0.f ? 0.f : 1.f / total[nt];
            __bf16 *out = (__bf16 *)a.out + (s.tok0 + tok[nt]) * a.out_st + hq[nt] * a.out_sh;
#pragma unroll
            for (int t = 0; t < VT; ++t)
                if (16 * t < D)
                    store4(out + 16 * t + 4 * g, o[t][nt][0] * inv, o[t][nt][1] * inv, o[t][nt][2] * inv, o[t][nt][3] * inv);
        } else {
            const int64_t at = ((tile * a.cache.heads + head) * a.splits + split) * ROWS + nt * 16 + col;
#pragma unroll
            for (int t = 0; t < VT; ++t)
                if (16 * t < D) *reinterpret_cast<v4f *>(a.part + at * D + 16 * t + 4 * g) = o[t][nt];
            if (g == 0) {
                a.stat[2 * at] = most[nt] * sm.c;
                a.stat[2 * at + 1] = total[nt];
            }
        }
    }
}

// Joins the splits of a query row: one wave a row, two dims a lane
template <int ROWS>
__global__ __launch_bounds__(256) void attention_join_kernel(const CachedArgs a)
{
    const int group = a.heads_q / a.cache.heads, D = a.cache.dim, lane = threadIdx.x & 63;
    const int r = (blockIdx.x % (ROWS / 4)) * 4 + (threadIdx.x >> 6);
    const int64_t rest = blockIdx.x / (ROWS / 4);
    const int head = (int)(rest % a.cache.heads);
    const int64_t tile = rest / a.cache.heads;
    Span s;
    int rt;
    const int b = find_unit(a.seq, a.cache.page_blocks * kBlockTokens, tile,
                            [&](const Span &x) { return (int)(((int64_t)x.n * group + ROWS - 1) / ROWS); }, s, rt);
    if (b < 0) return;
    const int64_t i = (int64_t)rt * ROWS + r;
    if (i >= (int64_t)s.n * group) return;
    const int64_t at = (tile * a.cache.heads + head) * a.splits * ROWS + r;
    float most = -INFINITY;
    for (int k = lane; k < a.splits; k += 64) most = fmaxf(most, a.stat[2 * (at + (int64_t)k * ROWS)]);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
    float total = 0.f, x0 = 0.f, x1 = 0.f;
    for (int k = 0; k < a.splits; ++k) {
        const int64_t e = at + (int64_t)k * ROWS;
        const float l = a.stat[2 * e + 1], y = a.stat[2 * e];
        if (l == 0.f) continue;
        const float f = y == most ? 1.f : __builtin_amdgcn_exp2f(y - most);
        total += l * f;
        if (2 * lane < D) {
            const v2f v = *reinterpret_cast<const v2f *>(a.part + e * D + 2 * lane);
            x0 += v[0] * f;
            x1 += v[1] * f;
        }
    }
    if (2 * lane >= D) return;
    const float inv = total == 0.f ? 0.f : 1.f / total;
    __bf16 *out = (__bf16 *)a.out + (s.tok0 + i / group) * a.out_st + (head * group + (int)(i % group)) * a.out_sh;
    *reinterpret_cast<bf16x2v *>(out + 2 * lane) = bf16x2v{(__bf16)(x0 * inv), (__bf16)(x1 * inv)};
}

template <int DT, int MODS, int NT>
hipError_t launch(const CachedArgs &a, hipStream_t stream)
{
    const int64_t heads = a.tiles * a.cache.heads, n = heads * a.splits;
    if (n > INT32_MAX || heads * (4 * NT) > INT32_MAX) return hipErrorInvalidConfiguration;
    attention_cached_kernel<DT, MODS, NT><<<(uint32_t)n, 256, 0, stream>>>(a);
    if (a.splits > 1) attention_join_kernel<16 * NT><<<(uint32_t)(heads * 4 * NT), 256, 0, stream>>>(a);
    return hipGetLastError();
}

template <int DT, int NT>
hipError_t launch_mods(const CachedArgs &a, hipStream_t stream)
{
    switch ((a.mask.cap > 0.f ? 1 : 0) | (a.mask.slopes ? 2 : 0)) {
    case 0: return launch<DT, 0, NT>(a, stream);
    case 1: return launch<DT, 1, NT>(a, stream);
    case 2: return launch<DT, 2, NT>(a, stream);
    default: return launch<DT, 3, NT>(a, stream);
    }
}

}  // namespace

hipError_t launch_attention_cached(const CachedArgs &a, hipStream_t stream)
{
    if (a.tiles == 0) return hipSuccess;
    if (a.cache.dim <= 64) return a.wide ? launch_mods<64, 4>(a, stream) : launch_mods<64, 1>(a, stream);
    return a.wide ? launch_mods<128, 4>(a, stream) : launch_mods<128, 1>(a, stream);
}

}  // namespace q2d
