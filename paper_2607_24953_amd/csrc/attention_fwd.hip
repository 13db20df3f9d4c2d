// Attention forward: O = softmax(S) V over the pairs that the masks leave, one pass over
// the keys with the running maximum and sum of each row.
//
// A wave owns 32 queries.  S^T = K Q^T puts a query's scores into one lane pair (see
// attention_common.hpp), where the maximum and the sum are register reductions and one
// exchange; O^T += V^T P^T takes P^T from those registers.  Keys and values stream through
// the LDS stages of stages_of() (global_load_lds, the next tiles on their way while one is used).
//
// Two roundings besides the result's: for bfloat16 operands, P to bfloat16 (to nearest even; the
// matrix cores take no float32 beside bfloat16), which is off by up to 2^-8 of a weight, while the
// sum that divides takes the unrounded weights; and there is none for float32.  Scores, maxima,
// sums and O are float32 throughout.
//
// What bounds it.  bfloat16, 128 dims: a 32 x 32 tile of scores is 16 MFMAs of 32 cycles
// beside the exponentials, maximum, sum and rounding of 16 scores a lane, which two waves a SIMD
// lay over one another, but not without gaps: 4 x 4096 tokens, 32 heads, causal 0.64 to 0.68 ms
// (810 to 860 TFLOP/s; matrix unit busy for 37 % of the time, vector unit 42 %), without causal order
// 950 to 990, where a library's product of 8192 x 8192 x 8192 reaches 1157; the causal loss is
// workgroups of unequal length at the end.  A cap adds a second exponential and a reciprocal a
// score: 16384 tokens, 32 on 8 heads, window of 4096: 1.42 ms, 680 TFLOP/s, vector unit busy for
// 68 %, matrix unit 28 %.  64 dims have half the products for the same softmax, and in documents
// workgroups of unequal length: 16384 tokens in ten documents, 32 on 8 heads: 0.40 ms, 425 TFLOP/s
// (tiles that documents cut counted for what is seen of them), vector unit 42 %, matrix unit 18 %,
// and 40 % of the waves' cycles waiting.  float32: the float32 matrix rate (153 TFLOP/s) and, in
// the NARROW form, one wave a SIMD that waits for its only LDS stage: 3 x 777 queries on 1999 keys,
// 6 on 2 heads, 72 dims in documents 0.18 ms, 26 TFLOP/s.
#include "attention_common.hpp"

namespace q2d {

namespace {

// A workgroup of four waves owns 128
// queries and its waves share tiles of 64 (float32: 32) keys; or (NARROW) 32 queries, and
// each wave takes its quarter of tiles of 128 keys, joined at the end.  DC is 64, 96 or 128: dims
// round up to whole 32s of O's tiles (fewer than 33 run as 64).  Three waves a SIMD where their
// registers allow it (64 dims, bfloat16).
template <typename T, int DC, int MODS, bool NARROW>
__global__ __launch_bounds__(256, DC <= 64 && sizeof(T) == 2 && !NARROW ? 3 : NARROW ? 1 : 2)
void attention_fwd_kernel(const AttentionArgs a)
{
    constexpr bool CAP = MODS & 1, BIAS = MODS & 2, F32 = sizeof(T) == 4;
    // DC dims are computed (a multiple of 32, dim rounded up), DT lie in an LDS row
    constexpr int DT = DC <= 64 ? 64 : 128, KS = DC / 16, DS = DC / 32;
    constexpr int NW = 4, BM = NARROW ? 32 : 32 * NW, BN = NARROW ? 32 * NW : F32 ? 32 : 64, WN = NARROW ? 32 : BN;
    typedef Tile<T, DT> Lds;
    constexpr int kBytes = BN * Lds::kRowBytes, NS = stages_of(2 * kBytes);
    __shared__ __align__(1024) uint8_t smem[NS][2][kBytes];
    __shared__ __align__(16) int32_t doc_of[NS][BN < 64 ? 64 : BN];   // documents of a tile's keys
    __shared__ uint32_t found[NW][BN / 32];                    // rows with infinities and NaN
    __shared__ float stat[2][NW][32];                          // maxima and sums of the waves

    const AttentionMask &m = a.mask;
    const uint32_t tiles = (a.len_q + BM - 1) / BM;
    uint32_t head, qt;
    head_tile(blockIdx.x, gridDim.x, tiles, head, qt);
    qt = tiles - 1 - qt;                       // with causal order the longest rows go first
    const int b = head / a.heads_q, hq = head % a.heads_q, hk = hq / (a.heads_q / a.heads_kv);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, col = lane & 31;
    const int shift = a.len_k - a.len_q, D = a.dim;
    const int i0 = qt * BM, iw = NARROW ? i0 : i0 + wave * 32, i = iw + col;
    const int jw = NARROW ? 32 * wave : 0;                     // the wave's first key of a tile
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
    const float thr = 8.f / sm.c;
    const Sight sight = query_sight(m, p, a.len_k, prefix, my_doc);

    int end = (a.len_k + BN - 1) / BN;
    if (m.causal && !m.prefix) end = p1 < 0 ? 0 : min(end, p1 / BN + 1);
    auto see = [&](int t, Seen &g, Seen &w) __attribute__((always_inline)) {
        const int j0 = t * BN, j1 = min(j0 + BN, a.len_k) - 1, k0 = j0 + jw, k1 = min(k0 + WN, a.len_k) - 1;
        g = classify(m, prefix, p0, p1, j0, j1, dg, docs ? range_of(ranges, j0, j1) : Documents{});
        g.all = g.all && j0 + BN <= a.len_k;                   // (the copies behind the last key are masked)
        if (pw1 >= pw0 && k1 >= k0) {
            w = classify(m, prefix, pw0, pw1, k0, k1, dw, docs ? range_of(ranges, k0, k1) : Documents{});
            w.all = w.all && k0 + WN <= a.len_k;
        }
    };
    if (D < DT) {
        Lds::template clear<NW * 64>(smem[0][0], sizeof(smem));
        __syncthreads();
    }
    v16f o[DS] = {};
    float mx = -INFINITY, sum = 0.f;

    auto tile = [&](const Visit &at, int stage) __attribute__((always_inline)) {
        const int j0 = at.tile * BN + jw;
        const uint32_t kr = Lds::row_base(smem[stage][0] + jw * Lds::kRowBytes, lane);
        const uint32_t vc = Lds::column_base(smem[stage][1] + jw * Lds::kRowBytes, lane);
        // Operands are read from LDS kAhead products before they are used, those of the first
        // value products before the softmax.  In this order (pinned) 128 dims run 5-10 % faster
        // than in the compiler's; with 64 dims it costs registers, and the third wave of a SIMD
        // with them (10 % slower).
        constexpr int TN = WN / 32, kScores = TN * KS, kValues = TN * 2 * DS, kAhead = F32 ? 2 : DC <= 64 ? 1 : 6;
        Frag<T> ring[kAhead];
        auto read = [&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value, x = i - kScores;
            if constexpr (i < kScores) ring[i % kAhead] = Lds::row_frag(kr, i % TN, i / TN);
            else if constexpr (x < kValues) ring[i % kAhead] = Lds::column_frag(vc, 16 * (x / DS), x % DS);
        };
        v16f z[TN] = {};
        unroll<kAhead>(read);
        unroll<kScores>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            z[i % TN] = mma(ring[i % kAhead], qf[i / TN], z[i % TN]);
            read(std::integral_constant<int, i + kAhead>{});
            pin<(DC > 64)>();
        });
        if constexpr (CAP || BIAS) {
            const float d0 = (float)(p - j0 - 4 * h);        // (positions do not fit float32)
#pragma unroll
            for (int t = 0; t < WN / 32; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float x = z[t][r];
                    if constexpr (CAP) x = tanh_of<F32, MODS>(x * sm.k1);
                    if constexpr (BIAS) x = fmaf(-sm.slope, fabsf(d0 - (float)(32 * t + tile_row(r, 0))), x);
                    z[t][r] = x;
                }
        }
        if (!at.all) {
#pragma unroll
            for (int t = 0; t < WN / 32; ++t) {
                const uint32_t w = sight.word(j0 + 32 * t, docs && !at.same ? &doc_of[stage][jw + 32 * t] : nullptr) >> (4 * h);
#pragma unroll
                for (int r = 0; r < 16; ++r) z[t][r] = word_bit(w, r) ? z[t][r] : -INFINITY;
            }
        }
        float top = z[0][0];
#pragma unroll
        for (int t = 0; t < WN / 32; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, z[t][r]);
        top = fmaxf(top, __shfl_xor(top, 32));
        // The running maximum moves only where it has been passed by 2^8: exponents up to
        // 8 above it are as good, and most tiles leave the sums as they are.
        if (__any(top > mx + thr)) {
            const float now = fmaxf(mx, top);
            const float f = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((mx - now) * sm.c);
#pragma unroll
            for (int dt = 0; dt < DS; ++dt) o[dt] *= f;
            sum *= f;
            mx = now;
        }
        const float base = mx == -INFINITY ? 0.f : mx;
        const float off = -base * sm.c;
#pragma unroll
        for (int t = 0; t < WN / 32; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float e = F32 ? (z[t][r] - base) * sm.c : fmaf(z[t][r], sm.c, off);
                z[t][r] = __builtin_amdgcn_exp2f(e);
                sum += z[t][r];
            }
        Frag<T> pf;
        unroll<kValues>([&](auto xc) __attribute__((always_inline)) {
            constexpr int x = decltype(xc)::value, i = kScores + x;
            if constexpr (x % DS == 0) pf = to_frag<T>(z[x / (2 * DS)], x / DS % 2);
            o[x % DS] = mma(ring[i % kAhead], pf, o[x % DS]);
            read(std::integral_constant<int, i + kAhead>{});
            pin<(DC > 64)>();
        });
    };
    auto check = [&](const Visit &at, int stage) __attribute__((always_inline)) {
        uint32_t bad[BN / 32], some = 0;
        non_finite<Lds, BN, NW>(smem[stage][1], &found[0][0], bad);
#pragma unroll
        for (int t = 0; t < BN / 32; ++t) some |= bad[t];
        if (!some) return;
        if (at.any) {
            const uint32_t vc = Lds::column_base(smem[stage][1] + jw * Lds::kRowBytes, lane);
#pragma unroll 1
            for (int t = 0; t < WN / 32; ++t) {
                const uint32_t w = sight.word(at.tile * BN + jw + 32 * t, docs && !at.same ? &doc_of[stage][jw + 32 * t] : nullptr);
                add_non_finite<T, DC, DT>(o, at.all ? ~0u : w, vc, 32 * t, h);
            }
        }
        Lds::template clean<BN, NW * 64>(smem[stage][1]);
    };
    auto fetch = [&](int stage, int t) __attribute__((always_inline)) {
        Lds::template load<BN, NW * 64>(smem[stage][0], k, a.k.sl, t * BN, a.len_k, D);
        Lds::template load<BN, NW * 64>(smem[stage][1], v, a.v.sl, t * BN, a.len_k, D);
        if (docs && wave < (BN + 63) / 64) load_words64(&doc_of[stage][64 * wave], docs, t * BN + 64 * wave, a.len_k);
    };
    tile_loop<NS, 2 * kBytes / (NW * 1024)>(end, see, fetch, check, tile);

    sum += __shfl_xor(sum, 32);
    if constexpr (NARROW) {
        // the four waves' rows on a common maximum
        if (h == 0) {
            stat[0][wave][col] = mx;
            stat[1][wave][col] = sum;
        }
        __syncthreads();                       // (and no wave reads a tile any more)
        float most = -INFINITY, total = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) most = fmaxf(most, stat[0][w][col]);
        auto weight = [&](float x, float l) {
            // (a sum of nothing counts 0, one that is NaN stays)
            return l == 0.f ? 0.f : x == most ? 1.f : __builtin_amdgcn_exp2f((x - most) * sm.c);
        };
#pragma unroll
        for (int w = 0; w < NW; ++w) total += weight(stat[0][w][col], stat[1][w][col]) * stat[1][w][col];
        const float f = weight(mx, sum);
#pragma unroll
        for (int dt = 0; dt < DS; ++dt) o[dt] *= f;
        join_waves<DS>(o, smem[0][0]);
        if (wave != 0) return;
        mx = most;
        sum = total;
    }
    if (!row) return;
    // (a row that sees keys sees its own position, or keys below and beside it; of scores that are
    // all -infinity the softmax is NaN)
    const bool sees = docs ? my_doc >= 0 : p >= 0 || prefix > 0 || sight.hi > max(sight.lo, 0);
    if (sum == 0.f && sees) sum = __builtin_nanf("");
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T *out = (T *)a.out.p + b * a.out.sb + (int64_t)i * a.out.sl + hq * a.out.sh;
    store_columns<T, DS>(out, o, inv, h, D);
    if (a.lse && h == 0)
        a.lse[((int64_t)b * a.heads_q + hq) * a.len_q + i] =
            sum == 0.f ? -INFINITY : (mx * sm.c + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <typename T, int DC, int MODS>
hipError_t launch(const AttentionArgs &a, hipStream_t stream)
{
    const int64_t heads = (int64_t)a.heads_q * a.batch, n = heads * ((a.len_q + 127) / 128);
    // 32 rows a workgroup where 128 would leave compute units without one: 128 tokens, 4 heads,
    // 64 dims, float32, forward and backward 79 -> 50 us; 3 x 777 queries on 1999 keys, 6 heads,
    // 72 dims, float32 676 -> 174 us.  With a workgroup of 128 rows for each compute unit the
    // narrow form loses, its tiles being shared by no one: bfloat16, 128 dims 62 us against 86.
    const bool narrow = n < kComputeUnits;
    const int64_t grid = narrow ? heads * ((a.len_q + 31) / 32) : n;
    if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
    if (narrow) attention_fwd_kernel<T, DC, MODS, true><<<(uint32_t)grid, 256, 0, stream>>>(a);
    else attention_fwd_kernel<T, DC, MODS, false><<<(uint32_t)grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

template <typename T, int DC>
hipError_t launch_mods(const AttentionArgs &a, hipStream_t stream)
{
    constexpr bool f32 = sizeof(T) == 4;
    switch (mods_of(a.mask, f32)) {
    case 0: return launch<T, DC, 0>(a, stream);
    case 1: return launch<T, DC, 1>(a, stream);
    case 2: return launch<T, DC, 2>(a, stream);
    case 3: return launch<T, DC, 3>(a, stream);
    default: return launch<T, DC, f32 ? 3 : kAnyCap>(a, stream);
    }
}

template <typename T>
hipError_t launch_dims(const AttentionArgs &a, hipStream_t stream)
{
    if (a.dim <= 64) return launch_mods<T, 64>(a, stream);
    return a.dim <= 96 ? launch_mods<T, 96>(a, stream) : launch_mods<T, 128>(a, stream);
}

}  // namespace

hipError_t launch_attention_fwd(const AttentionArgs &a, bool f32, hipStream_t stream)
{
    if (a.mask.documents) {
        const hipError_t e = launch_document_ranges(a, stream);
        if (e != hipSuccess) return e;
    }
    return f32 ? launch_dims<float>(a, stream) : launch_dims<__bf16>(a, stream);
}

}  // namespace q2d
