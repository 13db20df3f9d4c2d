// Attention forward: O = softmax(S) V over the pairs that the masks leave, one pass over
// the keys with the running maximum and sum of each row.
//
// A wave owns 32 queries.  S^T = K Q^T puts a query's scores into one lane pair (see
// attention_common.hpp), where the maximum and the sum are register reductions and one
// exchange; O^T += V^T P^T takes P^T from those registers.  Keys and values stream through
// two LDS stages (global_load_lds, the next tile on its way while this one is used).
#include "attention_common.hpp"

namespace q2d {

namespace {

// MODS bit 0: capped scores, bit 1: distance bias
template <typename T, int DT, int MODS, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attention_fwd_kernel(const AttentionArgs a)
{
    constexpr int BN = sizeof(T) == 2 ? 64 : 32, BM = 32 * NW, KS = DT / 16, DS = DT / 32;
    constexpr bool CAP = MODS & 1, BIAS = MODS & 2, F32 = sizeof(T) == 4;
    typedef Tile<T, DT> Lds;
    __shared__ __align__(1024) uint8_t smem[2][2][BN * Lds::kRowBytes];
    __shared__ __align__(16) int32_t doc_of[2][64];            // documents of a tile's keys
    __shared__ uint32_t found[NW][BN / 32];                    // rows with infinities and NaN

    const AttentionMask &m = a.mask;
    const uint32_t tiles = (a.len_q + BM - 1) / BM;
    uint32_t head, qt;
    head_tile(blockIdx.x, gridDim.x, tiles, head, qt);
    qt = tiles - 1 - qt;                       // with causal order the longest rows go first
    const int b = head / a.heads_q, hq = head % a.heads_q, hk = hq / (a.heads_q / a.heads_kv);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, col = lane & 31;
    const int shift = a.len_k - a.len_q, D = a.dim;
    const int i0 = qt * BM, iw = i0 + wave * 32, i = iw + col;
    const int p = i + shift;
    const bool row = i < a.len_q;

    const T *q = (const T *)a.q.p + b * a.q.sb + (int64_t)i * a.q.sl + hq * a.q.sh;
    const T *k = (const T *)a.k.p + b * a.k.sb + hk * a.k.sh;
    const T *v = (const T *)a.v.p + b * a.v.sb + hk * a.v.sh;
    Frag<T> qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = global_frag<T>(q, row, ks, h, D);

    const int prefix = m.prefix ? min(max(m.prefix[b], 0), a.len_k) : 0;
    const int32_t *docs = m.documents ? m.documents + (int64_t)b * a.len_k : nullptr;
    const int2 *ranges = a.ranges + (int64_t)b * ((a.len_k + 63) / 64);
    const int p0 = i0 + shift, p1 = min(i0 + BM, a.len_q) - 1 + shift;
    const int pw0 = iw + shift, pw1 = min(iw + 32, a.len_q) - 1 + shift;
    Documents dg = {}, dw = {};
    int my_doc = 0;
    if (docs) {
        dg = range_of(ranges, p0, p1);
        if (pw1 >= pw0) dw = range_of(ranges, pw0, pw1);
        my_doc = row && p >= 0 ? docs[p] : -1;
    }
    const ScoreMap sm = score_map(m, hq);
    const float thr = 8.f / sm.c, pos = (float)p;
    const Sight sight = query_sight(m, p, a.len_k, prefix, my_doc);

    int end = (a.len_k + BN - 1) / BN;
    if (m.causal && !m.prefix) end = p1 < 0 ? 0 : min(end, p1 / BN + 1);
    auto see = [&](int t, Seen &g, Seen &w) {
        const int j0 = t * BN, j1 = min(j0 + BN, a.len_k) - 1;
        const Documents dk = docs ? range_of(ranges, j0, j0) : Documents{};
        g = classify(m, prefix, p0, p1, j0, j1, dg, dk);
        if (pw1 >= pw0) {
            w = classify(m, prefix, pw0, pw1, j0, j1, dw, dk);
            w.all = w.all && j0 + BN <= a.len_k;
        }
    };

    if (D < DT) {
        Lds::template clear<NW * 64>(smem[0][0], sizeof(smem));
        __syncthreads();
    }
    v16f o[DS] = {};
    float mx = -INFINITY, sum = 0.f;

    // one tile of keys; all: no pair of this wave is masked
    auto tile = [&](bool all, int stage, int j0) __attribute__((always_inline)) {
        const uint8_t *kt = smem[stage][0], *vt = smem[stage][1];
        const uint32_t kr = Lds::row_base(kt, lane), vc = Lds::column_base(vt, lane);
        v16f z[BN / 32] = {};
#pragma unroll
        for (int t = 0; t < BN / 32; ++t)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) z[t] = mma(Lds::row_frag(kr, t, ks), qf[ks], z[t]);
        if constexpr (CAP || BIAS) {
            const float d0 = pos - (float)j0 - (float)(4 * h);
#pragma unroll
            for (int t = 0; t < BN / 32; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float x = z[t][r];
                    if constexpr (CAP) x = tanh_of(x * sm.k1, F32);
                    if constexpr (BIAS) x = fmaf(-sm.slope, fabsf(d0 - (float)(32 * t + tile_row(r, 0))), x);
                    z[t][r] = x;
                }
        }
        if (!all) {
#pragma unroll
            for (int t = 0; t < BN / 32; ++t) {
                const uint32_t w = sight.word(j0 + 32 * t, docs ? &doc_of[stage][32 * t] : nullptr) >> (4 * h);
#pragma unroll
                for (int r = 0; r < 16; ++r) z[t][r] = word_bit(w, r) ? z[t][r] : -INFINITY;
            }
        }
        float top = z[0][0];
#pragma unroll
        for (int t = 0; t < BN / 32; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, z[t][r]);
        top = fmaxf(top, __shfl_xor(top, 32));
        // The running maximum moves only where it has been passed by 2^8: exponents up to
        // 8 above it are as good, and most tiles leave the sums as they are.
        if (__any(top > mx + thr)) {
            const float now = fmaxf(mx, top);
            const float f = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mx - now) * sm.c);
#pragma unroll
            for (int dt = 0; dt < DS; ++dt) o[dt] *= f;
            sum *= f;
            mx = now;
        }
        const float base = mx == -INFINITY ? 0.f : mx;
        const float off = -base * sm.c;
#pragma unroll
        for (int t = 0; t < BN / 32; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float e = F32 ? (z[t][r] - base) * sm.c : fmaf(z[t][r], sm.c, off);
                z[t][r] = __builtin_amdgcn_exp2f(e);
                sum += z[t][r];
            }
#pragma unroll
        for (int t = 0; t < BN / 32; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const Frag<T> pf = to_frag<T>(z[t], s);
#pragma unroll
                for (int dt = 0; dt < DS; ++dt)
                    o[dt] = mma(Lds::column_frag(vc, 32 * t + 16 * s, dt), pf, o[dt]);
            }
    };
    auto check = [&](int stage, int j0, bool any, bool all) __attribute__((always_inline)) {
        uint32_t bad[BN / 32];
        non_finite<Lds, BN, NW>(smem[stage][1], &found[0][0], bad);
        uint32_t some = 0;
#pragma unroll
        for (int t = 0; t < BN / 32; ++t) some |= bad[t];
        if (!some) return;
        if (any) {
            const uint32_t vc = Lds::column_base(smem[stage][1], lane);
#pragma unroll 1
            for (int t = 0; t < BN / 32; ++t)
                add_non_finite<T, DT>(o, all ? ~0u : sight.word(j0 + 32 * t, docs ? &doc_of[stage][32 * t] : nullptr), vc,
                                      32 * t, h);
        }
        Lds::template clean<BN, NW * 64>(smem[stage][1]);
    };
    auto fetch = [&](int stage, int t) __attribute__((always_inline)) {
        Lds::template load<BN, NW * 64>(smem[stage][0], k, a.k.sl, t * BN, a.len_k, D);
        Lds::template load<BN, NW * 64>(smem[stage][1], v, a.v.sl, t * BN, a.len_k, D);
        if (docs && wave == 0) load_words64(doc_of[stage], docs, t * BN, a.len_k);
    };

    Schedule sched;
    int cur = sched.next(end, see), stage = 0;
    if (cur >= 0) fetch(0, cur);
    while (cur >= 0) {
        const bool part = sched.part, any = sched.wave_any, all = sched.wave_all;
        wait_vmcnt<0>();
        block_barrier();
        const int next = sched.next(end, see);
        if (next >= 0) fetch(stage ^ 1, next);
        if (part) check(stage, cur * BN, any, all);
        if (any) tile(all, stage, cur * BN);
        wait_lgkm();
        cur = next;
        stage ^= 1;
    }

    sum += __shfl_xor(sum, 32);
    if (!row) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T *out = (T *)a.out.p + b * a.out.sb + (int64_t)i * a.out.sl + hq * a.out.sh;
    store_columns<T, DS>(out, o, inv, h, D);
    if (a.lse && h == 0)
        a.lse[((int64_t)b * a.heads_q + hq) * a.len_q + i] =
            sum == 0.f ? -INFINITY : (mx * sm.c + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <typename T, int DT, int MODS, int NW>
hipError_t launch(const AttentionArgs &a, hipStream_t stream)
{
    const int64_t n = (int64_t)((a.len_q + 32 * NW - 1) / (32 * NW)) * a.heads_q * a.batch;
    if (n > INT32_MAX) return hipErrorInvalidConfiguration;
    attention_fwd_kernel<T, DT, MODS, NW><<<(uint32_t)n, NW * 64, 0, stream>>>(a);
    return hipGetLastError();
}

template <typename T, int DT>
hipError_t launch_mods(const AttentionArgs &a, hipStream_t stream)
{
    switch ((a.mask.cap > 0.f ? 1 : 0) | (a.mask.slopes ? 2 : 0)) {
    case 0: return launch<T, DT, 0, 4>(a, stream);
    case 1: return launch<T, DT, 1, 4>(a, stream);
    case 2: return launch<T, DT, 2, 4>(a, stream);
    default: return launch<T, DT, 3, 4>(a, stream);
    }
}

}  // namespace

hipError_t launch_attention_fwd(const AttentionArgs &a, bool f32, hipStream_t stream)
{
    if (a.mask.documents) {
        const hipError_t e = launch_document_ranges(a, stream);
        if (e != hipSuccess) return e;
    }
    if (f32) return a.dim <= 64 ? launch_mods<float, 64>(a, stream) : launch_mods<float, 128>(a, stream);
    return a.dim <= 64 ? launch_mods<__bf16, 64>(a, stream) : launch_mods<__bf16, 128>(a, stream);
}

}  // namespace q2d
