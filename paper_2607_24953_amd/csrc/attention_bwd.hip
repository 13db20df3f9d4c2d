// Attention backward.  With P = exp(S - lse), dP = dO V^T and delta = rowsum(dO * O):
//   dS = P (dP - delta) (1 - tanh^2 where scores are capped)
//   dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K.
// One kernel owns keys and sums dK and dV over the queries (of all query heads that share
// the key head), one owns queries and sums dQ over the keys.  Both form S and dP again:
// seven products in place of five, but every sum has one owner, so there are no atomics and
// the results do not depend on the order of workgroups.
//
// Roundings besides the results': for bfloat16 operands, P and dS to bfloat16 as operands of
// the second products (as P in the forward kernel; P to float16 on its way to dK, see
// attention_dkv_pair_kernel), and delta is formed from the stored O, which has been rounded to
// bfloat16: it shifts dP by up to 2^-8 of |dO||O| and saves a second copy of O in float32 (rows
// that see few keys, where it counts the most, have an exact one: exact_delta).  In units of
// rounding the exact gradient once, dV is off by 1.3 to 1.4 (its rounding and P's), dQ and dK by 1.4
// to 1.6, with a steep distance bias or interleaved documents up to 1.7 (their rounding, dS's, and
// delta): 0.0024 of their norm where one rounding is 0.0017.  For float32 there is none.
//
// As in the forward kernel, the first products leave the tile in the registers that the
// second ones take as operand: S, dP as [query][key] where keys are owned (columns), as
// [key][query] where queries are.
#include "attention_common.hpp"

namespace q2d {

namespace {

// Probabilities and dS are formed times 2^kShift, which the final scaling takes back exactly:
// where probabilities pass through LDS as float16 (attention_dkv_pair_kernel) all of those that
// count are then normal numbers, the largest below 2^16.
constexpr float kShift = 15.f, kUnshift = 1.f / 32768.f;

// sum over the 16 lanes of a row
__device__ __forceinline__ float row_sum(float s)
{
#pragma unroll
    for (int d = 1; d < 16; d *= 2) s += __shfl_xor(s, d);
    return s;
}

// Rows that may see no more than their own and the kNear - 1 positions before it: there delta as
// sum P dP, where these weights are all of the row's, in place of `rounded`, formed from the rounded
// O.  O's rounding enters dS as P r |dO||O|: little beside the rounding of a dS that is a
// sum over many keys, but all there is in a row of one key, whose dS is 0.  dQ's and dK's errors
// in units of rounding the exact result once: 600 tokens in documents of 1 to 33 tokens 1.73 ->
// 1.48, in longer ones 1.60 -> 1.49, in one 1.52 -> 1.46; the backward of 16384 tokens in ten
// documents, 64 dims, 0.96 -> 0.97 ms.  Rows whose few keys lie apart keep theirs.
constexpr int kNear = 8;

__device__ __forceinline__ float exact_delta(const AttentionArgs &a, int b, int i, int hq, int l, float lse2, float rounded)
{
    const AttentionMask &m = a.mask;
    const int p = i + a.len_k - a.len_q, D = a.dim, hk = hq / (a.heads_q / a.heads_kv);
    const int32_t *docs = m.documents ? m.documents + (int64_t)b * a.len_k : nullptr;
    if (p < 0 || !m.causal) return rounded;
    const int doc = docs ? docs[p] : 0;
    const bool few = p < kNear || (m.window && m.window <= kNear) || (docs && docs[p - kNear] != doc);
    if (!few || doc < 0) return rounded;
    const __bf16 *q = (const __bf16 *)a.q.p + b * a.q.sb + (int64_t)i * a.q.sl + hq * a.q.sh;
    const __bf16 *g = (const __bf16 *)a.dout.p + b * a.dout.sb + (int64_t)i * a.dout.sl + hq * a.dout.sh;
    const __bf16 *k = (const __bf16 *)a.k.p + b * a.k.sb + hk * a.k.sh, *v = (const __bf16 *)a.v.p + b * a.v.sb + hk * a.v.sh;
    const bool on = 8 * l < D;
    const bf16x8 qf = global_frag<__bf16>(q, on, l >> 1, l & 1, D), gf = global_frag<__bf16>(g, on, l >> 1, l & 1, D);
    const ScoreMap sm = score_map(m, hq);
    float mass = 0.f, sum = 0.f;
#pragma unroll 4
    for (int t = 0; t < kNear; ++t) {
        const int j = max(p - t, 0);
        const bool sees = p >= t && (!m.window || t < m.window) && (!docs || docs[j] == doc);
        const bf16x8 kf = global_frag<__bf16>(k + (int64_t)j * a.k.sl, on, l >> 1, l & 1, D);
        const bf16x8 vf = global_frag<__bf16>(v + (int64_t)j * a.v.sl, on, l >> 1, l & 1, D);
        float x = 0.f, dp = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x = fmaf((float)qf[e], (float)kf[e], x);
            dp = fmaf((float)gf[e], (float)vf[e], dp);
        }
        x = row_sum(x);
        dp = row_sum(dp);
        if (m.cap > 0.f) x = tanh_of<false, kAnyCap>(x * sm.k1);
        x = fmaf(-sm.slope, (float)t, x);
        const float w = __builtin_amdgcn_exp2f(fmaf(x, sm.c, -lse2));
        mass += sees ? w : 0.f;
        sum += sees ? w * dp : 0.f;
    }
    return mass >= 1.f - 0x1p-12f && fabsf(sum) < INFINITY ? sum / mass : rounded;
}

// delta of 4 rows a wave: 16 lanes a row.  Bound by memory: 4 x 4096 tokens, 32 heads of 128
// dims, bfloat16, 268 MB in 56 us (4.8 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void attention_delta_kernel(const AttentionArgs a)
{
    const int64_t rows = (int64_t)a.batch * a.heads_q * a.len_q;
    const int64_t r = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (r >= rows) return;
    const int l = threadIdx.x & 15;
    // neighbouring rows are neighbouring heads of a token
    const int hq = (int)(r % a.heads_q);
    const int64_t bl = r / a.heads_q;
    const int i = (int)(bl % a.len_q), b = (int)(bl / a.len_q);
    const T *o = (const T *)a.out.p + b * a.out.sb + (int64_t)i * a.out.sl + hq * a.out.sh;
    const T *g = (const T *)a.dout.p + b * a.dout.sb + (int64_t)i * a.dout.sl + hq * a.dout.sh;
    float s = 0.f;
    if (8 * l < a.dim) {
        const Frag<T> x = global_frag<T>(o, true, l >> 1, l & 1, a.dim);
        const Frag<T> y = global_frag<T>(g, true, l >> 1, l & 1, a.dim);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += (float)x[j] * (float)y[j];
    }
    s = row_sum(s);
    const int64_t at = ((int64_t)b * a.heads_q + hq) * a.len_q + i;
    const float lse2 = a.lse[at] * kLog2e;
    if constexpr (sizeof(T) == 2) s = exact_delta(a, b, i, hq, l, lse2, s);
    if (l != 0) return;
    a.delta[at] = s;
    a.lse2[at] = lse2 - kShift;
}

// Documents of 64 positions at a time (struct Documents): 16384 tokens 4 us, a launch
__global__ __launch_bounds__(64) void document_ranges_kernel(const int32_t *docs, int len, int2 *ranges)
{
    const int n = (len + 63) / 64, b = blockIdx.x / n, t = blockIdx.x % n, j = t * 64 + threadIdx.x;
    int lo = INT32_MAX, hi = -1;
    bool padding = false;
    if (j < len) {
        const int d = docs[(int64_t)b * len + j];
        padding = d < 0;
        if (!padding) lo = hi = d;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        lo = min(lo, __shfl_xor(lo, d));
        hi = max(hi, __shfl_xor(hi, d));
    }
    padding = __any(padding);
    if (threadIdx.x == 0) ranges[blockIdx.x] = make_int2(padding ? ~lo : lo, hi);
}

// ---------------------------------------------------------------- rows that are not finite
//
// Rows with an infinity or a NaN among their numbers, in tiles with masked pairs.  The products
// leave them out (`skip`); behind the loop, where its registers are free, the pairs that see
// them are added in plain arithmetic on the rows in memory.

// The tiles of a loop that have masked pairs, and their rows of x (and y) that are not finite:
// f(row), for a wave
template <int ROWS, int WIDTH, typename T, typename See, typename F>
__device__ __forceinline__ void add_rows(int end, See &&see, int first, int n, const T *x, int64_t sx, const T *y, int64_t sy,
                                         int D, F &&f)
{
    Schedule sched;
    for (Visit at = sched.take(end, see); at.tile >= 0; at = sched.take(end, see)) {
        if (!at.part || !at.any) continue;
        const int r0 = at.tile * ROWS + first, r1 = min(r0 + WIDTH, n);
#pragma unroll 1
        for (int r = r0; r < r1; ++r) {
            bool bad = false;
            for (int d = threadIdx.x & 63; d < D; d += 64)
                bad = bad || !(fabsf((float)x[r * sx + d]) < INFINITY) || !(fabsf((float)y[r * sy + d]) < INFINITY);
            if (__any(bad)) f(r);
        }
    }
}

// product of a lane pair's own row with a row that all lanes share, in both lanes
template <typename T>
__device__ __forceinline__ float row_dot(const T *own, bool valid, const T *row, int h, int D)
{
    float s = 0.f;
#pragma unroll 1
    for (int d = valid ? 8 * h : D; d < D; d += 16) {
        const Frag<T> x = global_frag<T>(own + d, true, 0, 0, 8), y = global_frag<T>(row + d, true, 0, 0, 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf((float)x[e], (float)y[e], s);
    }
    return s + __shfl_xor(s, 32);
}

struct PairWeights { float p, ds; };

// P and dS of a pair from its products q.k and dO.v and its distance
template <typename T, int MODS>
__device__ __forceinline__ PairWeights pair_weights(const ScoreMap &sm, float qk, float dp, int distance, float lse2, float delta)
{
    float u = 1.f;
    if constexpr (MODS & 1) {
        qk = tanh_of<sizeof(T) == 4, MODS>(qk * sm.k1);
        u = 1.f - qk * qk;
    }
    if constexpr (MODS & 2) qk = fmaf(-sm.slope, fabsf((float)distance), qk);
    const float p = __builtin_amdgcn_exp2f(fmaf(qk, sm.c, -lse2));
    return {p, p * (dp - delta) * u};
}

// accumulators (rows d, a column a lane pair) += w times a row of memory, in the columns that see it
template <typename T, int DS>
__device__ __forceinline__ void add_row(v16f *acc, const T *row, float w, bool sees, int h, int D)
{
#pragma unroll
    for (int dt = 0; dt < DS; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * dt + 8 * g + 4 * h;
            if (sees && d < D) {
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[dt][4 * g + i] = fmaf(w, (float)row[d + i], acc[dt][4 * g + i]);
            }
        }
}

// ---------------------------------------------------------------- dQ

// A workgroup's layout and NARROW are the forward kernel's.  Three products a tile, S, dP and
// dS K, all of 32 x 32 tiles with the row's numbers (lse, delta) in one lane pair.  Bound by the
// matrix cores with the exponentials between: 4 x 4096 tokens, 32 heads of 128 dims, causal,
// bfloat16 0.83 ms (990 TFLOP/s of its three products; matrix unit busy for 45 % of the time,
// vector unit 35 %); with a cap, 2 x 4096 tokens, 16 heads 0.32 ms (650; 27 and 48 %); 64 dims in
// documents (16384 tokens, 32 on 8 heads) 0.50 ms (500; 21 and 34 %, 42 % of the waves' cycles
// waiting).  128 dims spill five registers (20 bytes a lane), float32 with 128 dims 46 to 92.
template <typename T, int DC, int MODS, bool NARROW>
__global__ __launch_bounds__(256, NARROW ? 1 : 2) void attention_dq_kernel(const AttentionArgs a)
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

    const AttentionMask &m = a.mask;
    const uint32_t tiles = (a.len_q + BM - 1) / BM;
    uint32_t head, qt;
    head_tile(blockIdx.x, gridDim.x, tiles, head, qt);
    qt = tiles - 1 - qt;
    const int b = head / a.heads_q, hq = head % a.heads_q, hk = hq / (a.heads_q / a.heads_kv);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, col = lane & 31;
    const int shift = a.len_k - a.len_q, D = a.dim;
    const int i0 = qt * BM, iw = NARROW ? i0 : i0 + wave * 32, i = iw + col;
    const int jw = NARROW ? 32 * wave : 0;                     // the wave's first key of a tile
    const int p = i + shift;
    const bool row = i < a.len_q;

    const T *q = (const T *)a.q.p + b * a.q.sb + (int64_t)i * a.q.sl + hq * a.q.sh;
    const T *g = (const T *)a.dout.p + b * a.dout.sb + (int64_t)i * a.dout.sl + hq * a.dout.sh;
    const T *k = (const T *)a.k.p + b * a.k.sb + hk * a.k.sh;
    const T *v = (const T *)a.v.p + b * a.v.sb + hk * a.v.sh;
    Frag<T> qf[KS], gf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        qf[ks] = global_frag<T>(q, row, ks, h, D);
        gf[ks] = global_frag<T>(g, row, ks, h, D);
    }
    const int64_t at = ((int64_t)b * a.heads_q + hq) * a.len_q + i;
    // (rows outside: probabilities of 0)
    const float lse2 = row ? a.lse2[at] : INFINITY, delta = row ? a.delta[at] : 0.f;

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
    const Sight sight = query_sight(m, p, a.len_k, prefix, my_doc);

    int end = (a.len_k + BN - 1) / BN;
    if (m.causal && !m.prefix) end = p1 < 0 ? 0 : min(end, p1 / BN + 1);
    auto see = [&](int t, Seen &g, Seen &w) __attribute__((always_inline)) {
        const int j0 = t * BN, j1 = min(j0 + BN, a.len_k) - 1, k0 = j0 + jw, k1 = min(k0 + WN, a.len_k) - 1;
        g = classify(m, prefix, p0, p1, j0, j1, dg, docs ? range_of(ranges, j0, j1) : Documents{});
        g.all = g.all && j0 + BN <= a.len_k;
        if (pw1 >= pw0 && k1 >= k0) {
            w = classify(m, prefix, pw0, pw1, k0, k1, dw, docs ? range_of(ranges, k0, k1) : Documents{});
            w.all = w.all && k0 + WN <= a.len_k;
        }
    };
    if (D < DT) {
        Lds::template clear<NW * 64>(smem[0][0], sizeof(smem));
        __syncthreads();
    }
    v16f dq[DS] = {};

    uint32_t skip[WN / 32] = {};        // keys of the tile that the products leave out
    bool left_out = false;

    auto tile = [&](const Visit &at, int stage) __attribute__((always_inline)) {
        const int j0 = at.tile * BN + jw;
        const uint8_t *kt = smem[stage][0] + jw * Lds::kRowBytes, *vt = smem[stage][1] + jw * Lds::kRowBytes;
        const uint32_t kr = Lds::row_base(kt, lane), vr = Lds::row_base(vt, lane), kc = Lds::column_base(kt, lane);
        // the order of the reads as in the forward kernel; a step of 32 keys is 2 KS products for
        // S and dP and 2 DS for dQ
        constexpr int kFirst = 2 * KS, kStep = kFirst + 2 * DS, kAll = WN / 32 * kStep, kAhead = F32 ? 2 : DC <= 64 ? 1 : 6;
        Frag<T> ring[kAhead];
        auto read = [&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value, t = i / kStep, x = i % kStep, y = x - kFirst;
            if constexpr (i >= kAll) return;
            else if constexpr (x < kFirst) ring[i % kAhead] = Lds::row_frag(x % 2 ? vr : kr, t, x / 2);
            else ring[i % kAhead] = Lds::column_frag(kc, 32 * t + 16 * (y / DS), y % DS);
        };
        unroll<kAhead>(read);
        unroll<WN / 32>([&](auto tc) __attribute__((always_inline)) {
            constexpr int t = decltype(tc)::value;
            v16f z = {}, e = {};
            unroll<kFirst>([&](auto xc) __attribute__((always_inline)) {
                constexpr int x = decltype(xc)::value, i = t * kStep + x;
                if constexpr (x % 2) e = mma(ring[i % kAhead], gf[x / 2], e);
                else z = mma(ring[i % kAhead], qf[x / 2], z);
                read(std::integral_constant<int, i + kAhead>{});
                pin<(DC > 64)>();
            });
            const float d0 = (float)(p - (j0 + 32 * t) - 4 * h);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float x = z[r], u = 1.f;
                if constexpr (CAP) {
                    x = tanh_of<F32, MODS>(x * sm.k1);
                    u = 1.f - x * x;
                }
                if constexpr (BIAS) x = fmaf(-sm.slope, fabsf(d0 - (float)tile_row(r, 0)), x);
                const float pr = __builtin_amdgcn_exp2f(fmaf(x, sm.c, -lse2));
                e[r] = pr * (e[r] - delta) * u;
            }
            if (!at.all) {
                const uint32_t w =
                    (sight.word(j0 + 32 * t, docs && !at.same ? &doc_of[stage][jw + 32 * t] : nullptr) & ~skip[t]) >> (4 * h);
#pragma unroll
                for (int r = 0; r < 16; ++r) e[r] = word_bit(w, r) ? e[r] : 0.f;
            }
            Frag<T> ef;
            unroll<2 * DS>([&](auto yc) __attribute__((always_inline)) {
                constexpr int y = decltype(yc)::value, i = t * kStep + kFirst + y;
                if constexpr (y % DS == 0) ef = to_frag<T>(e, y / DS);
                dq[y % DS] = mma(ring[i % kAhead], ef, dq[y % DS]);
                read(std::integral_constant<int, i + kAhead>{});
                pin<(DC > 64)>();
            });
        });
    };
    auto check = [&](Visit &at, int stage) __attribute__((always_inline)) {
        uint32_t bad[BN / 32], some = 0;
        non_finite<Lds, BN, NW>(smem[stage][0], &found[0][0], bad);
#pragma unroll
        for (int t = 0; t < BN / 32; ++t) some |= bad[t];
#pragma unroll
        for (int t = 0; t < WN / 32; ++t) skip[t] = pick<BN / 32>(bad, NARROW ? wave : t);
        if (!some) return;
        at.all = false;
        left_out = true;
        Lds::template clean<BN, NW * 64>(smem[stage][0]);
    };
    auto fetch = [&](int stage, int t) __attribute__((always_inline)) {
        Lds::template load<BN, NW * 64>(smem[stage][0], k, a.k.sl, t * BN, a.len_k, D);
        Lds::template load<BN, NW * 64>(smem[stage][1], v, a.v.sl, t * BN, a.len_k, D);
        if (docs && wave < (BN + 63) / 64) load_words64(&doc_of[stage][64 * wave], docs, t * BN + 64 * wave, a.len_k);
    };
    tile_loop<NS, 2 * kBytes / (NW * 1024)>(end, see, fetch, check, tile);
    if (__builtin_expect(left_out, false))
        add_rows<BN, WN>(end, see, jw, a.len_k, k, a.k.sl, k, a.k.sl, D, [&](int j) __attribute__((always_inline)) {
            const T *kj = k + (int64_t)j * a.k.sl, *vj = v + (int64_t)j * a.v.sl;
            const float qk = row_dot(q, row, kj, h, D), dp = row_dot(g, row, vj, h, D);
            const bool sees = sight.sees(j, docs, docs ? docs[j] : 0);
            add_row<T, DS>(dq, kj, pair_weights<T, MODS>(sm, qk, dp, p - j, lse2, delta).ds, sees, h, D);
        });
    if constexpr (NARROW) {
        __syncthreads();                       // no wave reads a tile any more
        join_waves<DS>(dq, smem[0][0]);
        if (wave != 0) return;
    }
    if (!row) return;
    T *out = (T *)a.dq.p + b * a.dq.sb + (int64_t)i * a.dq.sl + hq * a.dq.sh;
    store_columns<T, DS>(out, dq, m.scale * kUnshift, h, D);
}

// ---------------------------------------------------------------- dK, dV

// One key's dK or dV: the gradient itself, or a split's part of it
template <typename T, int DS>
__device__ __forceinline__ void store_dkv(const AttentionArgs &a, bool dv, int split, int b, int j, int hk, const v16f *x, int h)
{
    if (a.splits > 1) {
        const int64_t at = ((((int64_t)(dv ? a.splits : 0) + split) * a.batch + b) * a.len_k + j) * a.heads_kv + hk;
        store_columns<float, DS>(a.part + at * a.dim, x, 1.f, h, a.dim);
        return;
    }
    const HeadsView &to = dv ? a.dv : a.dk;
    store_columns<T, DS>((T *)to.p + b * to.sb + (int64_t)j * to.sl + hk * to.sh, x, dv ? kUnshift : a.mask.scale * kUnshift, h, a.dim);
}

// Sums the splits' parts in order: 4 neighbouring dims a thread.  Bound by memory: 4 parts of
// 16384 keys, 8 heads of 64 dims, 302 MB in 49 us.
template <typename T>
__global__ __launch_bounds__(256) void attention_dkv_sum_kernel(const AttentionArgs a)
{
    const int64_t rows = (int64_t)a.batch * a.len_k * a.heads_kv, n = rows * (a.dim / 4);
    int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (x >= 2 * n) return;
    const bool dv = x >= n;
    x -= dv ? n : 0;
    const float *p = a.part + (dv ? (int64_t)a.splits * n * 4 : 0) + x * 4;
    v4f sum = *reinterpret_cast<const v4f *>(p);
    for (int s = 1; s < a.splits; ++s) sum += *reinterpret_cast<const v4f *>(p + (int64_t)s * n * 4);
    const int d = (int)(x % (a.dim / 4)) * 4;
    const int64_t r = x / (a.dim / 4);
    const int hk = (int)(r % a.heads_kv), j = (int)(r / a.heads_kv % a.len_k), b = (int)(r / a.heads_kv / a.len_k);
    const HeadsView &to = dv ? a.dv : a.dk;
    const float f = dv ? kUnshift : a.mask.scale * kUnshift;
    store4((T *)to.p + b * to.sb + (int64_t)j * to.sl + hk * to.sh + d, sum[0] * f, sum[1] * f, sum[2] * f, sum[3] * f);
}

// A workgroup of four waves owns 128 keys and its waves share tiles of 64 (float32: 32)
// queries; or (NARROW) 32 keys, and each wave takes its quarter of tiles of 128 queries.  The
// key's column lies in one lane pair; the queries' lse and delta come from LDS, four numbers a
// read.  With 64 dims K, V, dK and dV of 32 keys fit beside two waves a SIMD: 16384 tokens in
// ten documents, 32 on 8 heads, causal, bfloat16 0.65 ms (520 TFLOP/s of four products, for what is
// seen; vector unit busy for 34 % of the time, matrix unit 22 %, 44 % of the waves' cycles waiting:
// for the barrier of each tile, and at the end for workgroups of unequal length).
template <typename T, int DC, int MODS, bool NARROW>
__global__ __launch_bounds__(256, DC <= 64 && sizeof(T) == 2 && !NARROW ? 2 : 1) void attention_dkv_kernel(const AttentionArgs a)
{
    constexpr bool CAP = MODS & 1, BIAS = MODS & 2, F32 = sizeof(T) == 4;
    // DC dims are computed (a multiple of 32, dim rounded up), DT lie in an LDS row
    constexpr int DT = DC <= 64 ? 64 : 128, KS = DC / 16, DS = DC / 32;
    constexpr int NW = 4, BN = NARROW ? 32 : 32 * NW, BQ = NARROW ? 32 * NW : F32 ? 32 : 64, WQ = NARROW ? 32 : BQ;
    typedef Tile<T, DT> Lds;
    constexpr int kBytes = BQ * Lds::kRowBytes, NS = stages_of(2 * kBytes), kWords = BQ < 64 ? 64 : BQ;
    __shared__ __align__(1024) uint8_t smem[NS][2][kBytes];
    __shared__ __align__(16) float rows[NS][2][kWords];         // lse2, delta of a tile's queries
    __shared__ __align__(16) int32_t doc_of[NS][kWords];        // and their documents
    __shared__ uint32_t found[2][NW][BQ / 32];                 // rows with infinities and NaN

    const AttentionMask &m = a.mask;
    const uint32_t tiles = (a.len_k + BN - 1) / BN;
    uint32_t head, kt;
    head_tile(blockIdx.x, gridDim.x, tiles, head, kt);
    const int split = head % a.splits, b = head / a.splits / a.heads_kv, hk = head / a.splits % a.heads_kv;
    // this workgroup's query heads [first, last) of those that share the key head
    const int group = a.heads_q / a.heads_kv, each = (group + a.splits - 1) / a.splits;
    const int first = split * each, last = min(first + each, group);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, col = lane & 31;
    const int shift = a.len_k - a.len_q, D = a.dim;
    const int j0 = kt * BN, jw = NARROW ? j0 : j0 + wave * 32, j = jw + col;
    const int iw = NARROW ? 32 * wave : 0;                     // the wave's first query of a tile
    const bool key = j < a.len_k;

    const T *k = (const T *)a.k.p + b * a.k.sb + (int64_t)j * a.k.sl + hk * a.k.sh;
    const T *v = (const T *)a.v.p + b * a.v.sb + (int64_t)j * a.v.sl + hk * a.v.sh;
    Frag<T> kf[KS], vf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        kf[ks] = global_frag<T>(k, key, ks, h, D);
        vf[ks] = global_frag<T>(v, key, ks, h, D);
    }
    const int prefix = m.prefix ? min(max(m.prefix[b], 0), a.len_k) : 0;
    const int32_t *docs = m.documents ? m.documents + (int64_t)b * a.len_k : nullptr;
    const int2 *ranges = a.ranges + (int64_t)b * ((a.len_k + 63) / 64);
    const int j1 = min(j0 + BN, a.len_k) - 1, jw1 = min(jw + 32, a.len_k) - 1;
    Documents dg = {}, dw = {};
    int my_doc = 0;
    if (docs) {
        dg = range_of(ranges, j0, j1);
        if (jw1 >= jw) dw = range_of(ranges, jw, jw1);
        my_doc = key ? docs[j] : -1;
    }
    Sight sight = key_sight(m, j, a.len_k, prefix, my_doc);    // (queries end at position len_k)
    if (docs) sight.lo = max(sight.lo, 0);                     // (and have no document below 0)

    // tiles of query rows [t BQ, ..)
    const int end = (a.len_q + BQ - 1) / BQ;
    auto see = [&](int t, Seen &g, Seen &w) __attribute__((always_inline)) {
        const int i0 = t * BQ, i1 = min(i0 + BQ, a.len_q) - 1, k0 = i0 + iw, k1 = min(k0 + WQ, a.len_q) - 1;
        g = classify(m, prefix, i0 + shift, i1 + shift, j0, j1,
                     docs ? range_of(ranges, i0 + shift, i1 + shift) : Documents{}, dg);
        g.all = g.all && i0 + BQ <= a.len_q;
        if (jw1 >= jw && k1 >= k0) {
            w = classify(m, prefix, k0 + shift, k1 + shift, jw, jw1,
                         docs ? range_of(ranges, k0 + shift, k1 + shift) : Documents{}, dw);
            w.all = w.all && k0 + WQ <= a.len_q;
        }
    };
    if (D < DT) {
        Lds::template clear<NW * 64>(smem[0][0], sizeof(smem));
        __syncthreads();
    }
    v16f dk[DS] = {}, dv[DS] = {};
    uint32_t skip[WQ / 32] = {};        // queries of the tile that the products leave out
    bool left_out = false;
    for (int gh = first; gh < last; ++gh) {
        const int hq = hk * group + gh;
        const T *q = (const T *)a.q.p + b * a.q.sb + hq * a.q.sh;
        const T *g = (const T *)a.dout.p + b * a.dout.sb + hq * a.dout.sh;
        const float *lse = a.lse2 + ((int64_t)b * a.heads_q + hq) * a.len_q;
        const float *delta = a.delta + ((int64_t)b * a.heads_q + hq) * a.len_q;
        const ScoreMap sm = score_map(m, hq);
        auto tile = [&](const Visit &at, int stage) __attribute__((always_inline)) {
            const int i0 = at.tile * BQ + iw;
            const uint8_t *qt = smem[stage][0] + iw * Lds::kRowBytes, *gt = smem[stage][1] + iw * Lds::kRowBytes;
            const uint32_t qr = Lds::row_base(qt, lane), gr = Lds::row_base(gt, lane);
            const uint32_t qc = Lds::column_base(qt, lane), gc = Lds::column_base(gt, lane);
#pragma unroll
            for (int t = 0; t < WQ / 32; ++t) {
                v16f z = {}, e = {};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) z = mma(Lds::row_frag(qr, t, ks), kf[ks], z);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) e = mma(Lds::row_frag(gr, t, ks), vf[ks], e);
                const int p0 = i0 + 32 * t + shift;
                const float d0 = (float)(p0 + 4 * h - j);
#pragma unroll
                for (int x4 = 0; x4 < 4; ++x4) {
                    const v4f l4 = *reinterpret_cast<const v4f *>(&rows[stage][0][iw + 32 * t + tile_row(4 * x4, h)]);
                    const v4f e4 = *reinterpret_cast<const v4f *>(&rows[stage][1][iw + 32 * t + tile_row(4 * x4, h)]);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const int r = 4 * x4 + y;
                        float x = z[r], u = 1.f;
                        if constexpr (CAP) {
                            x = tanh_of<F32, MODS>(x * sm.k1);
                            u = 1.f - x * x;
                        }
                        if constexpr (BIAS) x = fmaf(-sm.slope, fabsf(d0 + (float)tile_row(r, 0)), x);
                        z[r] = __builtin_amdgcn_exp2f(fmaf(x, sm.c, -l4[y]));
                        e[r] = z[r] * (e[r] - e4[y]) * u;
                    }
                }
                if (!at.all) {
                    const uint32_t w =
                        (sight.word(p0, docs && !at.same ? &doc_of[stage][iw + 32 * t] : nullptr) & ~skip[t]) >> (4 * h);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        z[r] = word_bit(w, r) ? z[r] : 0.f;
                        e[r] = word_bit(w, r) ? e[r] : 0.f;
                    }
                }
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const Frag<T> pf = to_frag<T>(z, s), ef = to_frag<T>(e, s);
#pragma unroll
                    for (int dt = 0; dt < DS; ++dt) {
                        dv[dt] = mma(Lds::column_frag(gc, 32 * t + 16 * s, dt), pf, dv[dt]);
                        dk[dt] = mma(Lds::column_frag(qc, 32 * t + 16 * s, dt), ef, dk[dt]);
                    }
                }
            }
        };
        auto check = [&](Visit &at, int stage) __attribute__((always_inline)) {
            uint32_t bq[BQ / 32], bg[BQ / 32], some = 0;
            non_finite<Lds, BQ, NW>(smem[stage][0], &found[0][0][0], bq);
            non_finite<Lds, BQ, NW>(smem[stage][1], &found[1][0][0], bg);
#pragma unroll
            for (int t = 0; t < BQ / 32; ++t) {
                bq[t] |= bg[t];
                some |= bq[t];
            }
#pragma unroll
            for (int t = 0; t < WQ / 32; ++t) skip[t] = pick<BQ / 32>(bq, NARROW ? wave : t);
            if (!some) return;
            at.all = false;
            left_out = true;
            Lds::template clean<BQ, NW * 64>(smem[stage][0]);
            Lds::template clean<BQ, NW * 64>(smem[stage][1]);
        };
        // (numbers past the ends repeat the last: those rows are masked, and a position
        // below zero has no document)
        auto fetch = [&](int st, int t) __attribute__((always_inline)) {
            Lds::template load<BQ, NW * 64>(smem[st][0], q, a.q.sl, t * BQ, a.len_q, D);
            Lds::template load<BQ, NW * 64>(smem[st][1], g, a.dout.sl, t * BQ, a.len_q, D);
            // 64 numbers a wave: lse2 by the first waves, delta by the last
            constexpr int kW = kWords / 64;
            if (wave < kW) load_words64(&rows[st][0][64 * wave], lse, t * BQ + 64 * wave, a.len_q);
            const int w = NW - 1 - wave;
            if (w < kW) load_words64(&rows[st][1][64 * w], delta, t * BQ + 64 * w, a.len_q);
            if (docs && wave < kW) load_words64(&doc_of[st][64 * wave], docs, t * BQ + 64 * wave + shift, a.len_k);
        };
        tile_loop<NS, 2 * kBytes / (NW * 1024)>(end, see, fetch, check, tile);
        block_barrier();           // the next head's first tile takes stage 0
    }
    for (int gh = first; __builtin_expect(left_out, false) && gh < last; ++gh) {
        const int hq = hk * group + gh;
        const T *q = (const T *)a.q.p + b * a.q.sb + hq * a.q.sh;
        const T *g = (const T *)a.dout.p + b * a.dout.sb + hq * a.dout.sh;
        const int64_t at = ((int64_t)b * a.heads_q + hq) * a.len_q;
        const ScoreMap sm = score_map(m, hq);
        add_rows<BQ, WQ>(end, see, iw, a.len_q, q, a.q.sl, g, a.dout.sl, D, [&](int i) __attribute__((always_inline)) {
            const T *qi = q + (int64_t)i * a.q.sl, *gi = g + (int64_t)i * a.dout.sl;
            const float qk = row_dot(k, key, qi, h, D), dp = row_dot(v, key, gi, h, D);
            const PairWeights x = pair_weights<T, MODS>(sm, qk, dp, i + shift - j, a.lse2[at + i], a.delta[at + i]);
            const bool sees = sight.sees(i + shift, docs, docs ? docs[max(i + shift, 0)] : 0);
            add_row<T, DS>(dv, gi, x.p, sees, h, D);
            add_row<T, DS>(dk, qi, x.ds, sees, h, D);
        });
    }
    if constexpr (NARROW) {
        join_waves<DS>(dk, smem[0][0]);
        __syncthreads();
        join_waves<DS>(dv, smem[0][0]);
        if (wave != 0) return;
    }
    if (!key) return;
    store_dkv<T, DS>(a, false, split, b, j, hk, dk, h);
    store_dkv<T, DS>(a, true, split, b, j, hk, dv, h);
}

typedef _Float16 half2v __attribute__((ext_vector_type(2)));

// registers 8 s .. 8 s + 7 of an output tile as float16
__device__ __forceinline__ u4v to_half(const v16f &x, int s)
{
    u4v w;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        w[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{x[8 * s + 2 * j], x[8 * s + 2 * j + 1]}), half2v));
    return w;
}

// The same for bfloat16 with more than 64 dims, where the two accumulators of 32 keys and
// their K and V fragments take 192 registers: one wave a SIMD could hold them, and would then
// be bound by issuing one instruction after the other.  So two waves share 32 keys: the first
// keeps K and dV, forms S and P, and leaves P in LDS; the second keeps V and dK, forms dP and,
// one tile later, dS.  P passes in the registers' own order (operand fragments) as float16, with
// the cap's derivative multiplied in: as bfloat16 its rounding would add to that of dS (dK off by
// 0.0030 of its norm in place of 0.0024, 0.0017 of it the rounding of dK itself).
// Measured, 4 x 4096 tokens, 32 heads of 128 dims, causal: 1.43 to 1.5 ms, 730 to 770 TFLOP/s of its
// four products (matrix unit busy for 31 % of the time, vector unit 33 %); one wave for both, its
// products interleaved by hand, was slower at every size tried.  Waiting (37 % of the waves'
// cycles) is for the other wave at the barrier of each tile, and between the products.
template <int DC, int MODS>
__global__ __launch_bounds__(512, 2) void attention_dkv_pair_kernel(const AttentionArgs a)
{
    typedef __bf16 T;
    constexpr bool CAP = MODS & 1, BIAS = MODS & 2;
    constexpr int DT = 128, KS = DC / 16, DS = DC / 32, BQ = 64, NW = 8, BN = 128;
    typedef Tile<T, DT> Lds;
    __shared__ __align__(1024) uint8_t smem[3][2][BQ * Lds::kRowBytes];
    __shared__ u4v shared_p[2][4][BQ / 32][2][64];             // [tile parity][keys][rows][half][lane]
    __shared__ float shared_scale[2][4][BQ / 32][64];          // of a lane's sixteen of them
    __shared__ __align__(16) float rows[3][2][64];             // lse2, delta of a tile's queries
    __shared__ __align__(16) int32_t doc_of[3][64];            // and their documents
    __shared__ uint32_t found[2][NW][BQ / 32];                 // rows with infinities and NaN

    const AttentionMask &m = a.mask;
    const uint32_t tiles = (a.len_k + BN - 1) / BN;
    uint32_t head, kt;
    head_tile(blockIdx.x, gridDim.x, tiles, head, kt);
    const int split = head % a.splits, b = head / a.splits / a.heads_kv, hk = head / a.splits % a.heads_kv;
    // this workgroup's query heads [first, last) of those that share the key head
    const int group = a.heads_q / a.heads_kv, each = (group + a.splits - 1) / a.splits;
    const int first = split * each, last = min(first + each, group);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool second = wave >= 4;
    const int keys = wave & 3;
    const int h = lane >> 5, col = lane & 31;
    const int shift = a.len_k - a.len_q, D = a.dim;
    const int j0 = kt * BN, jw = j0 + keys * 32, j = jw + col;
    const bool key = j < a.len_k;

    // K rows for the first wave, V rows for the second
    const HeadsView &mine = second ? a.v : a.k;
    const T *kv = (const T *)mine.p + b * mine.sb + (int64_t)j * mine.sl + hk * mine.sh;
    Frag<T> f[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) f[ks] = global_frag<T>(kv, key, ks, h, D);
    const int prefix = m.prefix ? min(max(m.prefix[b], 0), a.len_k) : 0;
    const int32_t *docs = m.documents ? m.documents + (int64_t)b * a.len_k : nullptr;
    const int2 *ranges = a.ranges + (int64_t)b * ((a.len_k + 63) / 64);
    const int j1 = min(j0 + BN, a.len_k) - 1, jw1 = min(jw + 32, a.len_k) - 1;
    Documents dg = {}, dw = {};
    int my_doc = 0;
    if (docs) {
        dg = range_of(ranges, j0, j1);
        if (jw1 >= jw) dw = range_of(ranges, jw, jw1);
        my_doc = key ? docs[j] : -1;
    }
    Sight sight = key_sight(m, j, a.len_k, prefix, my_doc);    // (queries end at position len_k)
    if (docs) sight.lo = max(sight.lo, 0);                     // (and have no document below 0)

    const int end = (a.len_q + BQ - 1) / BQ;
    auto see = [&](int t, Seen &s, Seen &w) {
        const int p0 = t * BQ + shift, p1 = min(t * BQ + BQ, a.len_q) - 1 + shift;
        const Documents dq = docs ? range_of(ranges, p0, p1) : Documents{};
        s = classify(m, prefix, p0, p1, j0, j1, dq, dg);
        s.all = s.all && t * BQ + BQ <= a.len_q;
        if (jw1 >= jw) {
            w = classify(m, prefix, p0, p1, jw, jw1, dq, dw);
            w.all = w.all && t * BQ + BQ <= a.len_q;
        }
    };
    if (D < DT) {
        Lds::template clear<NW * 64>(smem[0][0], sizeof(smem));
        __syncthreads();
    }

    // the visited tiles of all query heads, in order
    struct At { int tile, head; bool part, any, all, same; };
    Schedule sched;
    int gh = first;
    auto advance = [&]() __attribute__((always_inline)) {
        int t = sched.next(end, see);
        while (t < 0 && ++gh < last) {
            sched = Schedule();
            t = sched.next(end, see);
        }
        return At{t, gh, sched.part, sched.wave_any, sched.wave_all, sched.wave_same};
    };
    auto fetch = [&](int st, const At &at) __attribute__((always_inline)) {
        const int hq = hk * group + at.head, i0 = at.tile * BQ;
        Lds::template load<BQ, NW * 64>(smem[st][0], (const T *)a.q.p + b * a.q.sb + hq * a.q.sh, a.q.sl, i0, a.len_q, D);
        Lds::template load<BQ, NW * 64>(smem[st][1], (const T *)a.dout.p + b * a.dout.sb + hq * a.dout.sh, a.dout.sl, i0,
                                        a.len_q, D);
        // (numbers past the ends repeat the last: those rows are masked)
        if (wave < 2)
            load_words64(rows[st][wave], (wave ? a.delta : a.lse2) + ((int64_t)b * a.heads_q + hq) * a.len_q, i0, a.len_q);
        if (docs && wave == 2) load_words64(doc_of[st], docs, i0 + shift, a.len_k);
    };
    uint32_t skip[BQ / 32] = {};        // queries of the tile that the products leave out
    bool left_out = false;
    auto check = [&](int stage, At &at) __attribute__((always_inline)) {
        uint32_t bq[BQ / 32], bg[BQ / 32], some = 0;
        non_finite<Lds, BQ, NW>(smem[stage][0], &found[0][0][0], bq);
        non_finite<Lds, BQ, NW>(smem[stage][1], &found[1][0][0], bg);
#pragma unroll
        for (int t = 0; t < BQ / 32; ++t) {
            skip[t] = bq[t] | bg[t];
            some |= skip[t];
        }
        if (!some) return;
        at.all = false;
        left_out = true;
        Lds::template clean<BQ, NW * 64>(smem[stage][0]);
        Lds::template clean<BQ, NW * 64>(smem[stage][1]);
    };

    // Both waves' steps of 32 queries are KS products with rows of one operand and 2 DS with
    // columns of the other; reads are kAhead products ahead, as in the forward kernel.
    constexpr int kStep = KS + 2 * DS, kAhead = 6;
    auto read_pair = [&](auto ic, Frag<T> *ring, uint32_t row, uint32_t column) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value, t = i / kStep, x = i % kStep, y = x - KS;
        if constexpr (i >= BQ / 32 * kStep) return;
        else if constexpr (x < KS) ring[i % kAhead] = Lds::row_frag(row, t, x);
        else ring[i % kAhead] = Lds::column_frag(column, 32 * t + 16 * (y / DS), y % DS);
    };
    // The first wave on a tile: P, and its product with dO
    auto probabilities = [&](v16f *acc, int stage, int parity, const At &at) __attribute__((always_inline)) {
        const uint32_t qr = Lds::row_base(smem[stage][0], lane), gc = Lds::column_base(smem[stage][1], lane);
        const ScoreMap sm = score_map(m, hk * group + at.head);
        Frag<T> ring[kAhead];
        auto read = [&](auto ic) __attribute__((always_inline)) { read_pair(ic, ring, qr, gc); };
        unroll<kAhead>(read);
        unroll<BQ / 32>([&](auto tc) __attribute__((always_inline)) {
            constexpr int t = decltype(tc)::value;
            v16f z = {};
            unroll<KS>([&](auto xc) __attribute__((always_inline)) {
                constexpr int x = decltype(xc)::value, i = t * kStep + x;
                z = mma(ring[i % kAhead], f[x], z);
                read(std::integral_constant<int, i + kAhead>{});
                pin();
            });
            const int p0 = at.tile * BQ + 32 * t + shift;
            const float d0 = BIAS ? (float)(p0 + 4 * h - j) : 0.f;
            v16f pu;                                     // P times the cap's derivative
#pragma unroll
            for (int x4 = 0; x4 < 4; ++x4) {
                const v4f l4 = *reinterpret_cast<const v4f *>(&rows[stage][0][32 * t + tile_row(4 * x4, h)]);
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int r = 4 * x4 + y;
                    float x = z[r], u = 1.f;
                    if constexpr (CAP) {
                        x = tanh_of<false, MODS>(x * sm.k1);
                        u = 1.f - x * x;
                    }
                    if constexpr (BIAS) x = fmaf(-sm.slope, fabsf(d0 + (float)tile_row(r, 0)), x);
                    z[r] = __builtin_amdgcn_exp2f(fmaf(x, sm.c, -l4[y]));
                    if constexpr (CAP) pu[r] = z[r] * u;
                }
            }
            if (!at.all) {
                const uint32_t w =
                    (sight.word(p0, docs && !at.same ? &doc_of[stage][32 * t] : nullptr) & ~skip[t]) >> (4 * h);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    z[r] = word_bit(w, r) ? z[r] : 0.f;
                    if constexpr (CAP) pu[r] = word_bit(w, r) ? pu[r] : 0.f;
                }
            }
            // A lane (a key) whose float16 numbers are all below the normal ones, while it sees
            // something: weights below 2^-29, all that a far key may have.  They pass times a
            // power of two, which the second wave takes back (4 x 4096 tokens, 32 heads of 128
            // dims: the whole backward 2.51 ms, 2.45 without).
            u4v half[2] = {to_half(CAP ? pu : z, 0), to_half(CAP ? pu : z, 1)};
            uint32_t bits = 0;
            float back = 1.f;
#pragma unroll
            for (int x = 0; x < 4; ++x) bits |= half[0][x] | half[1][x];
            if (__builtin_expect(__any((bits & 0x7c007c00u) == 0), false)) {
                float top = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, CAP ? pu[r] : z[r]);
                // (the largest to [2^14, 2^15))
                const int up = (bits & 0x7c007c00u) != 0 || top == 0.f ? 0 : min(141 - (int)(f_bits(top) >> 23), 126);
                const float f = bits_f((uint32_t)(127 + up) << 23);
                back = bits_f((uint32_t)(127 - up) << 23);
#pragma unroll
                for (int s = 0; s < 2; ++s) half[s] = to_half(CAP ? pu * f : z * f, s);
            }
            shared_scale[parity][keys][t][lane] = back;
#pragma unroll
            for (int s = 0; s < 2; ++s) shared_p[parity][keys][t][s][lane] = half[s];
            Frag<T> pf;
            unroll<2 * DS>([&](auto yc) __attribute__((always_inline)) {
                constexpr int y = decltype(yc)::value, i = t * kStep + KS + y, s = y / DS;
                if constexpr (y % DS == 0) pf = to_frag<T>(z, s);
                acc[y % DS] = mma(ring[i % kAhead], pf, acc[y % DS]);
                read(std::integral_constant<int, i + kAhead>{});
                pin();
            });
        });
    };
    // The second wave on the tile before: dS, and its product with Q
    auto gradients = [&](v16f *acc, int stage, int parity, const At &at) __attribute__((always_inline)) {
        const uint32_t gr = Lds::row_base(smem[stage][1], lane), qc = Lds::column_base(smem[stage][0], lane);
        Frag<T> ring[kAhead];
        auto read = [&](auto ic) __attribute__((always_inline)) { read_pair(ic, ring, gr, qc); };
        unroll<kAhead>(read);
        unroll<BQ / 32>([&](auto tc) __attribute__((always_inline)) {
            constexpr int t = decltype(tc)::value;
            v16f e = {};
            unroll<KS>([&](auto xc) __attribute__((always_inline)) {
                constexpr int x = decltype(xc)::value, i = t * kStep + x;
                e = mma(ring[i % kAhead], f[x], e);
                read(std::integral_constant<int, i + kAhead>{});
                pin();
            });
            u4v pw[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) pw[s] = shared_p[parity][keys][t][s][lane];
            const float back = shared_scale[parity][keys][t][lane];
            auto p_of = [&](int r) __attribute__((always_inline)) {
                const uint32_t w = pw[r / 8][r % 8 / 2];
                const half2v x = __builtin_bit_cast(half2v, w);
                return (float)(r % 2 ? x[1] : x[0]);
            };
#pragma unroll
            for (int x4 = 0; x4 < 4; ++x4) {
                const v4f e4 = *reinterpret_cast<const v4f *>(&rows[stage][1][32 * t + tile_row(4 * x4, h)]);
#pragma unroll
                for (int y = 0; y < 4; ++y) e[4 * x4 + y] = p_of(4 * x4 + y) * (e[4 * x4 + y] - e4[y]);
            }
            if (!at.all) {
                // (what is not seen may have brought a NaN into dP)
#pragma unroll
                for (int r = 0; r < 16; ++r) e[r] = p_of(r) != 0.f ? e[r] : 0.f;
            }
            if (__builtin_expect(__any(back != 1.f), false)) e *= back;
            Frag<T> ef;
            unroll<2 * DS>([&](auto yc) __attribute__((always_inline)) {
                constexpr int y = decltype(yc)::value, i = t * kStep + KS + y;
                if constexpr (y % DS == 0) ef = to_frag<T>(e, y / DS);
                acc[y % DS] = mma(ring[i % kAhead], ef, acc[y % DS]);
                read(std::integral_constant<int, i + kAhead>{});
                pin();
            });
        });
    };

    // (a loop for each of the two: they share nothing but the barriers)
    auto run = [&](auto second) __attribute__((always_inline)) {
        constexpr bool SECOND = decltype(second)::value;
        v16f acc[DS] = {};                               // dV, or dK
        At cur = advance(), before = {-1, 0, false, false, false, false};
        int stage = 0, parity = 0;
        if (cur.tile >= 0) fetch(0, cur);
        while (cur.tile >= 0 || before.tile >= 0) {
            // this tile is here, the last one's P too, and all waves are done with the one before
            wait_vmcnt<0>();
            wait_lgkm();
            block_barrier();
            At next = cur;
            if (cur.tile >= 0) {
                next = advance();
                if (next.tile >= 0) fetch(stage == 2 ? 0 : stage + 1, next);
                if (cur.part) check(stage, cur);
            }
            if constexpr (SECOND) {
                if (before.tile >= 0 && before.any) gradients(acc, stage == 0 ? 2 : stage - 1, parity ^ 1, before);
            } else {
                if (cur.tile >= 0 && cur.any) probabilities(acc, stage, parity, cur);
            }
            before = cur;
            cur = next;
            stage = stage == 2 ? 0 : stage + 1;
            parity ^= 1;
        }
        const T *kj = (const T *)a.k.p + b * a.k.sb + (int64_t)j * a.k.sl + hk * a.k.sh;
        const T *vj = (const T *)a.v.p + b * a.v.sb + (int64_t)j * a.v.sl + hk * a.v.sh;
        for (int gh = first; __builtin_expect(left_out, false) && gh < last; ++gh) {
            const int hq = hk * group + gh;
            const T *q = (const T *)a.q.p + b * a.q.sb + hq * a.q.sh;
            const T *g = (const T *)a.dout.p + b * a.dout.sb + hq * a.dout.sh;
            const int64_t at = ((int64_t)b * a.heads_q + hq) * a.len_q;
            const ScoreMap sm = score_map(m, hq);
            add_rows<BQ, BQ>(end, see, 0, a.len_q, q, a.q.sl, g, a.dout.sl, D, [&](int i) __attribute__((always_inline)) {
                const T *qi = q + (int64_t)i * a.q.sl, *gi = g + (int64_t)i * a.dout.sl;
                const float qk = row_dot(kj, key, qi, h, D), dp = SECOND ? row_dot(vj, key, gi, h, D) : 0.f;
                const PairWeights x = pair_weights<T, MODS>(sm, qk, dp, i + shift - j, a.lse2[at + i], a.delta[at + i]);
                const bool sees = sight.sees(i + shift, docs, docs ? docs[max(i + shift, 0)] : 0);
                add_row<T, DS>(acc, SECOND ? qi : gi, SECOND ? x.ds : x.p, sees, h, D);
            });
        }
        if (!key) return;
        store_dkv<T, DS>(a, !SECOND, split, b, j, hk, acc, h);
    };
    if (second) run(std::true_type{});
    else run(std::false_type{});
}

template <typename T, int DC, int MODS>
hipError_t launch(const AttentionArgs &a, hipStream_t stream)
{
    const int64_t hq = (int64_t)a.heads_q * a.batch, hk = (int64_t)a.heads_kv * a.batch * a.splits;
    int64_t nq = hq * ((a.len_q + 127) / 128), nk = hk * ((a.len_k + 127) / 128);
    // 32 rows a workgroup where 128 would leave compute units without one
    const bool narrow_q = nq < kComputeUnits, narrow_k = nk < kComputeUnits;
    if (narrow_q) nq = hq * ((a.len_q + 31) / 32);
    if (narrow_k) nk = hk * ((a.len_k + 31) / 32);
    if (nq > INT32_MAX || nk > INT32_MAX) return hipErrorInvalidConfiguration;
    if (narrow_k) attention_dkv_kernel<T, DC, MODS, true><<<(uint32_t)nk, 256, 0, stream>>>(a);
    else if constexpr (sizeof(T) == 2 && DC > 64) attention_dkv_pair_kernel<DC, MODS><<<(uint32_t)nk, 512, 0, stream>>>(a);
    else attention_dkv_kernel<T, DC, MODS, false><<<(uint32_t)nk, 256, 0, stream>>>(a);
    if (a.splits > 1) {
        const int64_t n = (int64_t)a.batch * a.len_k * a.heads_kv * (a.dim / 4) * 2;
        if ((n + 255) / 256 > INT32_MAX) return hipErrorInvalidConfiguration;
        attention_dkv_sum_kernel<T><<<(uint32_t)((n + 255) / 256), 256, 0, stream>>>(a);
    }
    if (narrow_q) attention_dq_kernel<T, DC, MODS, true><<<(uint32_t)nq, 256, 0, stream>>>(a);
    else attention_dq_kernel<T, DC, MODS, false><<<(uint32_t)nq, 256, 0, stream>>>(a);
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

hipError_t launch_document_ranges(const AttentionArgs &a, hipStream_t stream)
{
    const int64_t n = (int64_t)a.batch * ((a.len_k + 63) / 64);
    if (n > INT32_MAX) return hipErrorInvalidConfiguration;
    document_ranges_kernel<<<(uint32_t)n, 64, 0, stream>>>(a.mask.documents, a.len_k, a.ranges);
    return hipGetLastError();
}

hipError_t launch_attention_bwd(const AttentionArgs &a, bool f32, hipStream_t stream)
{
    if (a.mask.documents) {
        const hipError_t e = launch_document_ranges(a, stream);
        if (e != hipSuccess) return e;
    }
    const int64_t rows = ((int64_t)a.batch * a.heads_q * a.len_q + 15) / 16;
    if (rows > INT32_MAX) return hipErrorInvalidConfiguration;
    if (f32) attention_delta_kernel<float><<<(uint32_t)rows, 256, 0, stream>>>(a);
    else attention_delta_kernel<__bf16><<<(uint32_t)rows, 256, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return f32 ? launch_dims<float>(a, stream) : launch_dims<__bf16>(a, stream);
}

}  // namespace q2d
