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
// through a second kernel.  64 sequences of 600 to 8160 tokens, 32 on 8 heads of 128 dims: 557 MB
// in 123 us (4.5 TB/s, where a large copy moves 4.9 and a library's sum reads 4.0), and 11 us
// for the join; one sequence of 4097 tokens, whose bytes are 2 us: 10 and 5 us, latencies of a
// few dependent loads and of two launches.
//
// P is rounded to bfloat16 (to nearest even) as in the forward kernel on whole sequences; keys
// and values are exact, and sums are float32, in the workspace as well.
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

// Work is handed out per key head in units: a tile of ROWS query rows of a sequence (row r of it
// is token r / group, query head r % group) and one of `parts` equal shares of the super-blocks
// that the tile sees.  A sequence's tiles have as many parts as its length asks for, so that
// long and short sequences of a call end together: with W super-blocks to visit over all tiles,
// a part has about W / a.units of them, and at least kLeast.
template <int ROWS>
constexpr int kLeast = ROWS == 16 ? 4 : 8;

struct Place {
    int b, rt, head, part, parts, rows, prefix, p0, p1, from, to;
    int64_t unit;                  // number of the unit (BY_TILE: of the tile's first)
    Span s;
};

// Unit (BY_TILE: tile) `index` of a head; false: past the last.  One full wave, the same in all lanes.
template <int ROWS, bool BY_TILE>
__device__ __forceinline__ bool find_place(const CachedArgs &a, int group, int64_t index, Place &w)
{
    const AttentionMask &m = a.mask;
    const SequencesView &q = a.seq;
    const int lane = threadIdx.x & 63, page = a.cache.page_blocks * kBlockTokens;
    auto tiles_of = [&](const Span &x) { return (int)(((int64_t)x.n * group + ROWS - 1) / ROWS); };
    auto blocks_of = [&](const Span &x) {
        const int64_t seen = m.window && !m.prefix ? min((int64_t)x.len, (int64_t)m.window + ROWS) : x.len;
        return (int)((seen + kSuper - 1) / kSuper);
    };
    // (the first 64 sequences' spans stay in registers over the two passes)
    Span first = {0, 0, 0};
    if (lane < q.batch) first = span_of(q, page, lane);
    int64_t share = INT32_MAX;
    if (a.units > 0) {
        int64_t work = (int64_t)tiles_of(first) * blocks_of(first);
        for (int b = 64 + lane; b < q.batch; b += 64) {
            const Span x = span_of(q, page, b);
            work += (int64_t)tiles_of(x) * blocks_of(x);
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) work += __shfl_xor(work, d);
        share = max((work + a.units - 1) / a.units, (int64_t)kLeast<ROWS>);
    }
    int64_t carry = 0, units = 0;
    for (int base = 0; base < q.batch; base += 64) {
        const int b = base + lane;
        Span x = first;
        if (base > 0) {
            x = {0, 0, 0};
            if (b < q.batch) x = span_of(q, page, b);
        }
        const int tiles = tiles_of(x);
        const int parts = (int)min(max((blocks_of(x) + share - 1) / share, (int64_t)1), (int64_t)kMaxSplits);
        const int64_t all = (int64_t)tiles * parts, count = BY_TILE ? tiles : all;
        int64_t upto = count, units_upto = all;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t below = __shfl_up(upto, d);
            if (lane >= d) upto += below;
            if constexpr (BY_TILE) {
                const int64_t y = __shfl_up(units_upto, d);
                if (lane >= d) units_upto += y;
            }
        }
        const uint64_t past = __ballot(carry + upto > index);
        if (past) {
            const int at = __builtin_ctzll(past);
            w.b = base + at;
            w.s.n = __builtin_amdgcn_readlane(x.n, at);
            w.s.len = __builtin_amdgcn_readlane(x.len, at);
            w.s.tok0 = (int64_t)uniform64(__shfl((uint64_t)x.tok0, at));
            w.parts = __builtin_amdgcn_readlane(parts, at);
            const int local = __builtin_amdgcn_readfirstlane((int)(index - carry - __shfl(upto - count, at)));
            w.rt = BY_TILE ? local : local / w.parts;
            w.part = BY_TILE ? 0 : local % w.parts;
            w.unit = index;
            if (BY_TILE) w.unit = (int64_t)uniform64((uint64_t)(units + __shfl(units_upto - all, at))) + (int64_t)w.rt * w.parts;
            w.rows = min(ROWS, (int)((int64_t)w.s.n * group - (int64_t)w.rt * ROWS));
            return true;
        }
        carry += __shfl(upto, 63);
        if constexpr (BY_TILE) units += __shfl(units_upto, 63);
    }
    return false;
}

// The unit of this workgroup, and its super-blocks [from, to)
template <int ROWS>
__device__ __forceinline__ bool place_of(const CachedArgs &a, int group, Place &w)
{
    const AttentionMask &m = a.mask;
    if (!find_place<ROWS, false>(a, group, blockIdx.x / a.cache.heads, w)) return false;
    w.head = blockIdx.x % a.cache.heads;
    w.prefix = m.prefix ? min(max(m.prefix[w.b], 0), w.s.len) : 0;
    w.p0 = w.s.len - w.s.n + w.rt * ROWS / group;
    w.p1 = w.s.len - w.s.n + (w.rt * ROWS + w.rows - 1) / group;
    // tokens that some row sees: [t0, t1)
    int t1 = max(min(w.p1 + 1, w.s.len), w.prefix), t0 = m.window && !w.prefix ? max(w.p0 - m.window + 1, 0) : 0;
    if (t1 < t0) t1 = t0;
    const int sb0 = t0 / kSuper, sbs = (t1 + kSuper - 1) / kSuper - sb0;
    w.from = sb0 + (int)((int64_t)sbs * w.part / w.parts);
    w.to = sb0 + (int)((int64_t)sbs * (w.part + 1) / w.parts);
    return true;
}

// rows of no sequence: zeros (whoever works on the whole tensor next, as in blocks of rows that share
// a scale, would otherwise meet what the memory held)
__device__ __forceinline__ void clear_outside(const CachedArgs &a)
{
    const Outside x = outside_of(a.seq);
    const int64_t first = (int64_t)(blockIdx.x - a.grid) * 256 + threadIdx.x, step = (int64_t)(gridDim.x - a.grid) * 256;
    __bf16 *out = (__bf16 *)a.out;
    zero_rows(out, a.out_st, a.out_sh, x.lo, a.heads_q, a.cache.dim, first, step);
    zero_rows(out + x.hi * a.out_st, a.out_st, a.out_sh, a.seq.tokens - x.hi, a.heads_q, a.cache.dim, first, step);
}

template <int DT, int MODS>
__global__ __launch_bounds__(256, 2) void attention_cached_kernel(const CachedArgs a)
{
    if (blockIdx.x >= (uint32_t)a.grid) return clear_outside(a);
    constexpr bool CAP = MODS & 1, BIAS = MODS & 2;
    constexpr int KS = DT / 32, VT = DT / 16, ROWS = 16;
    // two waves' sums [row][dim] at a time, and all waves' statistics
    __shared__ __align__(16) float osum[2][ROWS * DT];
    __shared__ float stat[2][4][ROWS];

    const AttentionMask &m = a.mask;
    const int group = a.heads_q / a.cache.heads, D = a.cache.dim;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    Place w;
    if (!place_of<ROWS>(a, group, w)) return;
    const Span &s = w.s;

    // this lane's query row
    const int r = w.rt * ROWS + col, tok = r / group, hq = w.head * group + r % group, pos = s.len - s.n + tok;
    const bool row = col < w.rows;
    const ScoreMap sm = score_map(m, row ? hq : 0);
    bf16x8 qf[KS];
    const __bf16 *q = (const __bf16 *)a.q + (s.tok0 + tok) * a.q_st + hq * a.q_sh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        // the order of dims in which a 16-byte load of codes serves two steps
        const int d = 64 * (ks >> 1) + 16 * g + 8 * (ks & 1);
        bf16x8 x = {};
        if (row && d < D) x = *reinterpret_cast<const bf16x8 *>(q + d);
        qf[ks] = x;
    }
    const Sight sight = query_sight(m, pos, s.len, w.prefix, 0);

    v4f o[VT] = {};
    float mx = -INFINITY, sum = 0.f;
    const float thr = 8.f / sm.c;

    Codes<DT> c;
    Where ahead = {-1, -1};
    int sb = w.from + wave;
    if (sb < w.to) fetch<DT>(a, locate(a, w.b, w.head, sb, s.len, lane), lane, c);
    if (sb + 4 < w.to) ahead = locate(a, w.b, w.head, sb + 4, s.len, lane);
    for (; sb < w.to; sb += 4) {
        Codes<DT> next;
        if (sb + 4 < w.to) fetch<DT>(a, ahead, lane, next);
        if (sb + 8 < w.to) ahead = locate(a, w.b, w.head, sb + 8, s.len, lane);

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
        const bool all = j0 + kSuper - 1 <= w.p0 && j0 + kSuper <= s.len && (!m.window || w.p1 - j0 < m.window) &&
                         !__any(c.vs == kNoBlock);
        bf16x8 pf[2];
        v4f z[4] = {};
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int t = 0; t < DT / 64; ++t) {
                const u4v w = c.k[u][t];
                z[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_to_bf16(w[0], w[1], 1.f), qf[2 * t], z[u], 0, 0, 0);
                z[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_to_bf16(w[2], w[3], 1.f), qf[2 * t + 1], z[u], 0, 0, 0);
            }
        const int jl = j0 + 16 * g;
        const float d0 = (float)(pos - jl);
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x = z[u][i] * ks;
                if constexpr (CAP) x = tanh_of<false, MODS>(x);
                if constexpr (BIAS) x = fmaf(-sm.slope, fabsf(d0 - (float)(4 * u + i)), x);
                z[u][i] = x;
            }
        if (!all) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = jl + 4 * u + i;
                    const bool ok = ((j >= sight.lo && j < sight.hi) || j < w.prefix) && c.vs != kNoBlock;
                    z[u][i] = ok ? z[u][i] : -INFINITY;
                }
        }
        // A value scale of 255 marks a block with a NaN: rows that see it become NaN, however small
        // their weight of it (the maximum passes NaN scores over)
        if (__any(c.vs == 255)) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (c.vs == 255 && z[u][i] != -INFINITY) z[u][i] = __builtin_nanf("");
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, z[u][i]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        // (as in the forward kernel: the maximum moves only where it is passed by 2^8)
        if (__any(top > mx + thr)) {
            const float now = fmaxf(mx, top);
            const float f = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mx - now) * sm.c);
#pragma unroll
            for (int t = 0; t < VT; ++t) o[t] *= f;
            sum *= f;
            mx = now;
        }
        const float off = mx == -INFINITY ? 0.f : -mx * sm.c;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(fmaf(z[u][i], sm.c, off));
                sum += e;
                z[u][i] = e;
            }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) pf[k][i] = (__bf16)z[2 * k + (i >> 2)][i & 3];
        const float vs = bits_f((c.vs >= 255 ? 127u : c.vs) << 23);
#pragma unroll
        for (int t = 0; t < VT; ++t)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const bf16x8 x = fp8_to_bf16(c.v[t][2 * k], c.v[t][2 * k + 1], vs);
                o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, pf[k], o[t], 0, 0, 0);
            }
        c = next;
    }

    // join the four waves: common maximum, then the sums in two steps
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (g == 0) {
        stat[0][wave][col] = mx;
        stat[1][wave][col] = sum;
    }
    __syncthreads();
    float total = 0.f, most = -INFINITY;
#pragma unroll
    for (int x = 0; x < 4; ++x) most = fmaxf(most, stat[0][x][col]);
    auto weight = [&](float x, float l) {
        // (a sum of nothing counts 0, one that is NaN stays)
        return l == 0.f ? 0.f : x == most ? 1.f : __builtin_amdgcn_exp2f((x - most) * sm.c);
    };
#pragma unroll
    for (int x = 0; x < 4; ++x) total += weight(stat[0][x][col], stat[1][x][col]) * stat[1][x][col];
    const float f = weight(mx, sum);
#pragma unroll
    for (int t = 0; t < VT; ++t) o[t] *= f;
    auto put = [&](float *dst) {
#pragma unroll
        for (int t = 0; t < VT; ++t) *reinterpret_cast<v4f *>(dst + (t * 64 + lane) * 4) = o[t];
    };
    auto add = [&](const float *src) {
#pragma unroll
        for (int t = 0; t < VT; ++t) o[t] += *reinterpret_cast<const v4f *>(src + (t * 64 + lane) * 4);
    };
    if (wave >= 2) put(osum[wave - 2]);
    __syncthreads();
    if (wave < 2) add(osum[wave]);
    __syncthreads();
    if (wave == 1) put(osum[0]);
    __syncthreads();
    if (wave != 0 || !row) return;
    add(osum[0]);
    if (w.parts == 1) {
        const float inv = total == 0.f ? 0.f : 1.f / total;
        __bf16 *out = (__bf16 *)a.out + (s.tok0 + tok) * a.out_st + hq * a.out_sh;
#pragma unroll
        for (int t = 0; t < VT; ++t)
            if (16 * t < D) store4(out + 16 * t + 4 * g, o[t][0] * inv, o[t][1] * inv, o[t][2] * inv, o[t][3] * inv);
    } else {
        const int64_t at = (w.unit * a.cache.heads + w.head) * ROWS + col;
#pragma unroll
        for (int t = 0; t < VT; ++t)
            if (16 * t < D) *reinterpret_cast<v4f *>(a.part + at * D + 16 * t + 4 * g) = o[t];
        if (g == 0) {
            a.stat[2 * at] = most * sm.c;
            a.stat[2 * at + 1] = total;
        }
    }
}

// The same for prompts: 128 query rows a workgroup, 32 a wave, as in the forward kernel on whole
// sequences.  The workgroup converts each super-block once into LDS tiles of bfloat16 (exact:
// a code times its power of two), keys [token][dim] and values [dim][token], while the codes of
// the next one are on their way.  With the key rows taken in the order
// 16 (b / 2) + 8 h + 4 (b % 2) + i for output row 8 b + 4 h + i, a lane ends with 8 neighbouring
// tokens for each k-step, and value fragments are single 16-byte reads.
// Bound as the forward kernel is, with the conversion beside it: 4 prompts of 4096 tokens, 32
// heads of 128 dims 0.77 to 0.83 ms (660 to 710 TFLOP/s); capped, 12644 rows of 8 unequal
// sequences in 0.37 ms (460 TFLOP/s; vector unit busy for 58 % of the time, matrix unit 20 %).
template <int DC, int MODS>
__global__ __launch_bounds__(256, 2) void attention_cached_rows_kernel(const CachedArgs a)
{
    if (blockIdx.x >= (uint32_t)a.grid) return clear_outside(a);
    constexpr bool CAP = MODS & 1, BIAS = MODS & 2;
    constexpr int DT = DC <= 64 ? 64 : 128, KS = DC / 16, DS = DC / 32, ROWS = 128;
    constexpr int kPasses = kSuper * DT / (16 * 256);          // 16-byte loads of a thread, keys or values
    typedef Tile<__bf16, DT> Lds;
    __shared__ __align__(1024) uint8_t ktile[2][kSuper * DT * 2], vtile[2][kSuper * DT * 2];

    const AttentionMask &m = a.mask;
    const int group = a.heads_q / a.cache.heads, D = a.cache.dim;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, col = lane & 31;
    Place w;
    if (!place_of<ROWS>(a, group, w)) return;
    const Span &s = w.s;
    const int c = wave * 32 + col, r = w.rt * ROWS + c, tok = r / group, hq = w.head * group + r % group;
    const int pos = s.len - s.n + tok;
    const bool row = c < w.rows, some = wave * 32 < w.rows;
    // positions of the wave's first and last row
    const int pw0 = s.len - s.n + (w.rt * ROWS + wave * 32) / group;
    const int pw1 = s.len - s.n + (w.rt * ROWS + min(wave * 32 + 32, w.rows) - 1) / group;
    const ScoreMap sm = score_map(m, row ? hq : 0);
    const __bf16 *q = (const __bf16 *)a.q + (s.tok0 + tok) * a.q_st + hq * a.q_sh;
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = global_frag<__bf16>(q, row, ks, h, D);
    const Sight sight = query_sight(m, pos, s.len, w.prefix, 0);
    const float thr = 8.f / sm.c;

    // the two cache blocks of a super-block (-1: none), and their scale bytes
    struct Blocks {
        int64_t at[2];
        uint32_t ks[2], vs[2];
    };
    auto blocks_of = [&](int sb) __attribute__((always_inline)) {
        Blocks x;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x.at[i] = -1;
            x.ks[i] = 0;
            x.vs[i] = kNoBlock;
            const int blk = 2 * sb + i;
            if (sb < w.to && blk * kBlockTokens < s.len) x.at[i] = cache_block(a.cache, a.seq, w.b, blk, w.head);
            if (x.at[i] >= 0) {
                x.ks[i] = a.cache.ks[x.at[i]];
                x.vs[i] = a.cache.vs[x.at[i]];
            }
        }
        return x;
    };
    u4v kc[kPasses], vc[kPasses];
    auto fetch = [&](const Blocks &x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int slot = i * 256 + tid;
            // keys: 16 dims of a token; values: 16 tokens of a dim
            const int t = slot / (DT / 16), d = slot % (DT / 16) * 16;
            const int64_t kb = t < kBlockTokens ? x.at[0] : x.at[1];
            const int blk = slot / (2 * DT), dv = slot % (2 * DT) / 2;
            const int64_t vb = blk ? x.at[1] : x.at[0];
            kc[i] = vc[i] = u4v{0, 0, 0, 0};
            if (kb >= 0 && d < D)
                kc[i] = *reinterpret_cast<const u4v *>(a.cache.k + (kb * kBlockTokens + t % kBlockTokens) * D + d);
            if (vb >= 0 && dv < D)
                vc[i] = *reinterpret_cast<const u4v *>(a.cache.v + (vb * D + dv) * kBlockTokens + slot % 2 * 16);
        }
    };
    auto scale_of = [](uint32_t byte) { return bits_f((byte >= 255 ? 127u : byte) << 23); };
    // codes at hand (of super-block sb) -> bfloat16 tiles
    auto convert = [&](int stage, int sb, const Blocks &x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int slot = i * 256 + tid;
            const int t = slot / (DT / 16), c16 = slot % (DT / 16);
            const uint32_t kb = t < kBlockTokens ? x.ks[0] : x.ks[1];
            const float kscale = scale_of(kb);
            bf16x8 lo = fp8_to_bf16(kc[i][0], kc[i][1], kscale), hi = fp8_to_bf16(kc[i][2], kc[i][3], kscale);
            if (kb == 255) {
#pragma unroll
                for (int e = 0; e < 8; ++e) lo[e] = hi[e] = (__bf16)__builtin_nanf("");
            }
            *reinterpret_cast<bf16x8 *>(ktile[stage] + Lds::offset(t, 2 * c16)) = lo;
            *reinterpret_cast<bf16x8 *>(ktile[stage] + Lds::offset(t, 2 * c16 + 1)) = hi;

            const int blk = slot / (2 * DT), d = slot % (2 * DT) / 2, half = slot % 2;
            u4v v = vc[i];
            // tokens past the end: codes of 0 in place of what the page holds there
            const int n = s.len - (sb * kSuper + blk * kBlockTokens + half * 16);
            if (n < 16) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] &= (uint32_t)((1ull << (8 * min(max(n - 4 * e, 0), 4))) - 1);
            }
            const float vscale = scale_of(blk ? x.vs[1] : x.vs[0]);
            const int chunk = 4 * blk + 2 * half;
            uint8_t *p = vtile[stage] + d * (kSuper * 2);
            *reinterpret_cast<bf16x8 *>(p + ((chunk ^ ((d >> 1) & 7)) << 4)) = fp8_to_bf16(v[0], v[1], vscale);
            *reinterpret_cast<bf16x8 *>(p + (((chunk + 1) ^ ((d >> 1) & 7)) << 4)) = fp8_to_bf16(v[2], v[3], vscale);
        }
    };

    v16f o[DS] = {};
    float mx = -INFINITY, sum = 0.f;
    auto tile = [&](int stage, int sb, const Blocks &x) __attribute__((always_inline)) {
        const int j0 = sb * kSuper;
        if (j0 > pw1 && j0 >= w.prefix) return;
        const int krow = 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
        const uint32_t kr = Lds::fresh(Lds::address(ktile[stage]) + Lds::offset(krow, h));
        const uint32_t vr = Lds::fresh(Lds::address(vtile[stage]) + col * (kSuper * 2) + ((h ^ ((col >> 1) & 7)) << 4));
        // (reads ahead of the products as in the forward kernel)
        constexpr int kScores = 2 * KS, kValues = 4 * DS, kAhead = DC <= 64 ? 1 : 6;
        bf16x8 ring[kAhead];
        auto read = [&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value, y = i - kScores;
            if constexpr (i < kScores) ring[i % kAhead] = Lds::row_frag(kr, i % 2, i / 2);
            else if constexpr (y < kValues)
                ring[i % kAhead] = *Lds::template lds_ptr<bf16x8>((vr ^ (uint32_t)(2 * (y / DS) << 4)) + y % DS * 32 * kSuper * 2);
        };
        v16f z[2] = {};
        unroll<kAhead>(read);
        unroll<kScores>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            z[i % 2] = mma(ring[i % kAhead], qf[i / 2], z[i % 2]);
            read(std::integral_constant<int, i + kAhead>{});
            pin<(DC > 64)>();
        });
        // token of register i: 16 (i / 8) + 8 h + i % 8
        if constexpr (CAP || BIAS) {
            const float d0 = (float)(pos - j0 - 8 * h);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float y = z[t][i];
                    if constexpr (CAP) y = tanh_of<false, MODS>(y * sm.k1);
                    if constexpr (BIAS) y = fmaf(-sm.slope, fabsf(d0 - (float)(32 * t + 16 * (i >> 3) + (i & 7))), y);
                    z[t][i] = y;
                }
        }
        const bool all = j0 + kSuper - 1 <= pw0 && j0 + kSuper <= s.len && (!m.window || pw1 - j0 < m.window) &&
                         x.at[0] >= 0 && x.at[1] >= 0;
        if (!all) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t seen = x.at[t] >= 0 ? sight.word(j0 + 32 * t, nullptr) >> (8 * h) : 0u;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    z[t][i] = (seen >> (16 * (i >> 3) + (i & 7))) & 1 ? z[t][i] : -INFINITY;
            }
        }
        // (blocks with a NaN among the values, as in the kernel above)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (x.vs[t] == 255) {
#pragma unroll
                for (int i = 0; i < 16; ++i) z[t][i] = z[t][i] != -INFINITY ? __builtin_nanf("") : z[t][i];
            }
        }
        float top = z[0][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, z[t][i]);
        top = fmaxf(top, __shfl_xor(top, 32));
        // (as in the forward kernel: the maximum moves only where it is passed by 2^8)
        if (__any(top > mx + thr)) {
            const float now = fmaxf(mx, top);
            const float f = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((mx - now) * sm.c);
#pragma unroll
            for (int dt = 0; dt < DS; ++dt) o[dt] *= f;
            sum *= f;
            mx = now;
        }
        const float off = mx == -INFINITY ? 0.f : -mx * sm.c;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                z[t][i] = __builtin_amdgcn_exp2f(fmaf(z[t][i], sm.c, off));
                sum += z[t][i];
            }
        bf16x8 pf;
        unroll<kValues>([&](auto yc) __attribute__((always_inline)) {
            constexpr int y = decltype(yc)::value, i = kScores + y;
            if constexpr (y % DS == 0) pf = to_frag<__bf16>(z[y / (2 * DS)], y / DS % 2);
            o[y % DS] = mma(ring[i % kAhead], pf, o[y % DS]);
            read(std::integral_constant<int, i + kAhead>{});
            pin<(DC > 64)>();
        });
    };

    Blocks now = blocks_of(w.from), next = blocks_of(w.from + 1);
    if (w.from < w.to) {
        fetch(now);
        convert(0, w.from, now);
    }
    fetch(next);
    int stage = 0;
    for (int sb = w.from; sb < w.to; ++sb) {
        __syncthreads();
        Blocks after = next;
        if (sb + 1 < w.to) {
            after = blocks_of(sb + 2);
            convert(stage ^ 1, sb + 1, next);
            fetch(after);
        }
        if (some) tile(stage, sb, now);
        now = next;
        next = after;
        stage ^= 1;
    }

    sum += __shfl_xor(sum, 32);
    if (!row) return;
    if (w.parts == 1) {
        __bf16 *out = (__bf16 *)a.out + (s.tok0 + tok) * a.out_st + hq * a.out_sh;
        store_columns<__bf16, DS>(out, o, sum == 0.f ? 0.f : 1.f / sum, h, D);
    } else {
        const int64_t at = (w.unit * a.cache.heads + w.head) * ROWS + c;
        store_columns<float, DS>(a.part + at * D, o, 1.f, h, D);
        if (h == 0) {
            a.stat[2 * at] = mx * sm.c;
            a.stat[2 * at + 1] = sum;
        }
    }
}

// Joins the parts of a tile's query rows: two dims a lane, a wave takes kJoinRows rows of it.
// Bound by the latency of finding its tile (two scans over the sequences) and of one pass of
// loads: tiles of 16 rows one row a wave (64 sequences, 2048 rows of 128 dims: 11 us), tiles of
// 128 rows, where the finding counts more, four (8 unequal prompts, 12644 rows: the whole call
// 417 us with one, 384 with four, 387 with eight).
template <int ROWS>
constexpr int kJoinRows = ROWS == 16 ? 1 : 4;

template <int ROWS>
__global__ __launch_bounds__(256) void attention_join_kernel(const CachedArgs a)
{
    constexpr int kGroups = ROWS / (4 * kJoinRows<ROWS>);
    const int group = a.heads_q / a.cache.heads, D = a.cache.dim, lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t rest = blockIdx.x / kGroups;
    const int head = (int)(rest % a.cache.heads);
    Place w;
    if (!find_place<ROWS, true>(a, group, rest / a.cache.heads, w) || w.parts == 1) return;
    // (the host's bound, which offsets that do not ascend could pass)
    if (w.unit + w.parts > a.tiles + a.units) return;
    const int64_t step = (int64_t)a.cache.heads * ROWS;
#pragma unroll 2
    for (int n = 0; n < kJoinRows<ROWS>; ++n) {
        const int r = (blockIdx.x % kGroups * 4 + wave) * kJoinRows<ROWS> + n;
        if (r >= w.rows) return;
        const int64_t at = (w.unit * a.cache.heads + head) * ROWS + r;
        // lane k: part k's maximum and sum (there are at most kMaxSplits)
        float l = 0.f, y = -INFINITY;
        if (lane < w.parts) {
            const v2f x = *reinterpret_cast<const v2f *>(a.stat + 2 * (at + lane * step));
            y = x[0];
            l = x[1];
        }
        float most = y;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
        const float f = l == 0.f ? 0.f : y == most ? 1.f : __builtin_amdgcn_exp2f(y - most);
        float total = l * f, x0 = 0.f, x1 = 0.f;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
        const float *p = a.part + at * D + min(2 * lane, D - 2);
        // (a part without tokens has sums of 0, lanes past the last part a weight of 0)
        for (int k = 0; k < w.parts; k += 8) {
            v2f v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const v2f *>(p + min(k + i, w.parts - 1) * step * D);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float g = bits_f(__builtin_amdgcn_readlane(f_bits(f), k + i));
                x0 += v[i][0] * g;
                x1 += v[i][1] * g;
            }
        }
        const float inv = total == 0.f ? 0.f : 1.f / total;
        const int64_t i = (int64_t)w.rt * ROWS + r;
        __bf16 *out = (__bf16 *)a.out + (w.s.tok0 + i / group) * a.out_st + (head * group + (int)(i % group)) * a.out_sh;
        if (2 * lane < D) *reinterpret_cast<bf16x2v *>(out + 2 * lane) = bf16x2v{(__bf16)(x0 * inv), (__bf16)(x1 * inv)};
    }
}

// ROWS: query rows of a workgroup, 128 or 16
template <int DC, int MODS, int ROWS>
hipError_t launch(CachedArgs a, hipStream_t stream)
{
    // (every tile has a unit, and the parts of W / units super-blocks are no more than units)
    constexpr int groups = ROWS / (4 * kJoinRows<ROWS>);
    const int64_t tiles = a.tiles * a.cache.heads, units = (a.tiles + a.units) * a.cache.heads;
    const int64_t n = units + (a.seq.offsets ? zero_groups(a.seq.tokens) : 0);
    if (n > INT32_MAX || tiles * groups > INT32_MAX) return hipErrorInvalidConfiguration;
    a.grid = (int32_t)units;
    if constexpr (ROWS == 16) attention_cached_kernel<DC, MODS><<<(uint32_t)n, 256, 0, stream>>>(a);
    else attention_cached_rows_kernel<DC, MODS><<<(uint32_t)n, 256, 0, stream>>>(a);
    if (a.units > 0) attention_join_kernel<ROWS><<<(uint32_t)(tiles * groups), 256, 0, stream>>>(a);
    return hipGetLastError();
}

template <int DC, int ROWS>
hipError_t launch_mods(const CachedArgs &a, hipStream_t stream)
{
    switch (mods_of(a.mask, false)) {
    case 0: return launch<DC, 0, ROWS>(a, stream);
    case 1: return launch<DC, 1, ROWS>(a, stream);
    case 2: return launch<DC, 2, ROWS>(a, stream);
    case 3: return launch<DC, 3, ROWS>(a, stream);
    default: return launch<DC, kAnyCap, ROWS>(a, stream);
    }
}

}  // namespace

hipError_t launch_attention_cached(const CachedArgs &a, hipStream_t stream)
{
    if (a.tiles == 0) return hipSuccess;
    if (!a.wide) return a.cache.dim <= 64 ? launch_mods<64, 16>(a, stream) : launch_mods<128, 16>(a, stream);
    if (a.cache.dim <= 64) return launch_mods<64, 128>(a, stream);
    return a.cache.dim <= 96 ? launch_mods<96, 128>(a, stream) : launch_mods<128, 128>(a, stream);
}

}  // namespace q2d
