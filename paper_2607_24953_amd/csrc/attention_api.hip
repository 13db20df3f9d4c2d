// C ABI of the attention operators: argument validation, workspace layout and launches.
#include "q2d.h"
#include "attention.hpp"

#include <limits.h>
#include <math.h>

namespace {

using namespace q2d;

constexpr int64_t kMaxLen = int64_t(1) << 30;
constexpr int64_t kMaxPitch = int64_t(1) << 22;    // the tile loads' 32-bit row offsets

inline bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

// scale > 0, softcap >= 0; both within 2^-60 .. 2^60, where what the kernels form of them (their
// quotient, and scores' units by either) stays within float32
q2d_status check_scale(float scale, float softcap)
{
    if (!(scale > 0.f) || !isfinite(scale) || !(softcap >= 0.f) || !isfinite(softcap)) return Q2D_EINVAL;
    auto fits = [](float x) { return x >= 0x1p-60f && x <= 0x1p60f; };
    return fits(scale) && (softcap == 0.f || fits(softcap)) ? Q2D_OK : Q2D_EUNSUPPORTED;
}

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

// (an output's rows must not share memory: each stride passes what the smaller ones span)
q2d_status check_output(const q2d_heads &t, int64_t batch, int64_t length, int64_t heads, int64_t dim, int per)
{
    const q2d_status s = check_heads(t, batch, length, heads, dim, per);
    if (s != Q2D_OK) return s;
    struct { int64_t n, stride; } axis[3] = {{heads, t.stride_head}, {length, t.stride_length}, {batch, t.stride_batch}};
    auto order = [&](int i, int j) {
        if (axis[j].stride < axis[i].stride) { const auto x = axis[i]; axis[i] = axis[j]; axis[j] = x; }
    };
    for (auto &x : axis)
        if (x.n == 1) x.stride = 0;
    order(0, 1); order(1, 2); order(0, 1);
    int64_t span = dim;
    for (const auto &x : axis) {
        if (x.n == 1) continue;
        if (x.stride < span) return Q2D_EINVAL;
        span += (x.n - 1) * x.stride;
    }
    return Q2D_OK;
}

// A checked tensor's rows in memory: dim elements each, along up to three axes
struct Rows {
    uintptr_t at;
    int64_t n[3], s[3], dim, size;       // strides and dim in elements of `size` bytes, 0 for an extent of 1
};

Rows rows_of(const q2d_heads &t, int64_t batch, int64_t length, int64_t heads, int64_t dim, int per)
{
    Rows r = {reinterpret_cast<uintptr_t>(t.data), {batch, length, heads}, {t.stride_batch, t.stride_length, t.stride_head}, dim,
              16 / per};
    for (int i = 0; i < 3; ++i)
        if (r.n[i] == 1) r.s[i] = 0;
    return r;
}

// whether some row of b starts within dim of one of a: off + sum d[i] s[i] for d[i] in
// (-a.n[i], b.n[i]), the axes by falling stride (`axis`: the order)
bool rows_meet(const Rows &a, const Rows &b, const int64_t s[3], const int axis[3], int level, int64_t off)
{
    if (level == 3) return off > -a.dim && off < a.dim;
    const int i = axis[level];
    if (s[i] == 0) return rows_meet(a, b, s, axis, level + 1, off);
    // (smaller strides reach no further than this one)
    for (int64_t d = -off / s[i] - 1; d <= -off / s[i] + 1; ++d)
        if (d > -a.n[i] && d < b.n[i] && rows_meet(a, b, s, axis, level + 1, off + d * s[i])) return true;
    return false;
}

// Whether an output may share memory with another tensor of the call: rows of one system of
// strides between one another (heads of one tensor), or none.
bool apart(const Rows &a, const Rows &b)
{
    int64_t last_a = a.dim, last_b = b.dim, s[3];
    bool one = true;
    for (int i = 0; i < 3; ++i) {
        last_a += (a.n[i] - 1) * a.s[i];
        last_b += (b.n[i] - 1) * b.s[i];
        one = one && (a.s[i] == b.s[i] || a.n[i] == 1 || b.n[i] == 1);
        s[i] = a.n[i] == 1 ? b.s[i] : a.s[i];
    }
    if (a.at + last_a * a.size <= b.at || b.at + last_b * b.size <= a.at) return true;
    if (!one) return false;
    int axis[3] = {0, 1, 2};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (s[axis[j]] < s[axis[j + 1]]) { const int x = axis[j]; axis[j] = axis[j + 1]; axis[j + 1] = x; }
    return !rows_meet(a, b, s, axis, 0, ((int64_t)b.at - (int64_t)a.at) / a.size);
}

// the same rows: an output in the place of an input that only its own workgroup reads
bool same_rows(const Rows &a, const Rows &b)
{
    bool r = a.at == b.at;
    for (int i = 0; i < 3; ++i) r = r && a.n[i] == b.n[i] && a.s[i] == b.s[i];
    return r;
}

q2d_status check_sizes(const q2d_attention *a)
{
    if (!a) return Q2D_EINVAL;
    if (a->dtype != Q2D_F32 && a->dtype != Q2D_BF16) return Q2D_EINVAL;
    if ((a->causal != 0 && a->causal != 1) || a->batch <= 0 || a->heads_q <= 0 || a->heads_kv <= 0 || a->dim <= 0 ||
        a->len_q <= 0 || a->len_k <= 0 || a->window < 0)
        return Q2D_EINVAL;
    if (a->heads_q % a->heads_kv != 0) return Q2D_EINVAL;
    const q2d_status s = check_scale(a->scale, a->softcap);
    if (s != Q2D_OK) return s;
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

Rows query_rows(const q2d_attention *a, const q2d_heads &t)
{
    return rows_of(t, a->batch, a->len_q, a->heads_q, a->dim, a->dtype == Q2D_F32 ? 4 : 8);
}

Rows key_rows(const q2d_attention *a, const q2d_heads &t)
{
    return rows_of(t, a->batch, a->len_k, a->heads_kv, a->dim, a->dtype == Q2D_F32 ? 4 : 8);
}

HeadsView view(const q2d_heads &t) { return {t.data, t.stride_batch, t.stride_length, t.stride_head}; }

int64_t ranges_bytes(const q2d_attention *a)
{
    return a->documents ? up256((int64_t)a->batch * ((a->len_k + 63) / 64) * 8) : 0;
}

int64_t rows_bytes(const q2d_attention *a) { return up256((int64_t)a->batch * a->heads_q * a->len_q * 4); }

int64_t part_bytes(const q2d_attention *a)
{
    const int n = dkv_splits(a->batch, a->len_q, a->len_k, a->heads_q, a->heads_kv, a->documents != nullptr);
    return n > 1 ? up256((int64_t)n * a->batch * a->len_k * a->heads_kv * a->dim * 8) : 0;
}

int64_t workspace_of(const q2d_attention *a, bool backward)
{
    return ranges_bytes(a) + (backward ? 2 * rows_bytes(a) + part_bytes(a) : 0);
}

AttentionArgs make_args(const q2d_attention *a, void *workspace)
{
    AttentionArgs r = {};
    r.q = view(a->q); r.k = view(a->k); r.v = view(a->v); r.out = view(a->out);
    r.lse = a->lse;
    r.ranges = reinterpret_cast<int2 *>(workspace);
    r.delta = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(workspace) + ranges_bytes(a));
    r.lse2 = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(r.delta) + rows_bytes(a));
    r.mask.causal = a->causal;
    r.part = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(r.lse2) + rows_bytes(a));
    r.splits = dkv_splits(a->batch, a->len_q, a->len_k, a->heads_q, a->heads_kv, a->documents != nullptr);
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

inline bool on4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

q2d_status check_cache_sizes(const q2d_kv_cache &c)
{
    if (c.pages <= 0 || c.heads <= 0 || c.dim <= 0 || c.page_size <= 0 || c.page_size % 32 != 0) return Q2D_EINVAL;
    if (c.dim % 16 != 0 || c.dim > 128 || c.page_size > 65536 || c.heads > 16384) return Q2D_EUNSUPPORTED;
    int64_t blocks;
    if (__builtin_mul_overflow((int64_t)c.pages * c.heads, (int64_t)(c.page_size / 32), &blocks) || blocks > INT32_MAX)
        return Q2D_EUNSUPPORTED;
    return Q2D_OK;
}

q2d_status check_cache(const q2d_kv_cache *c)
{
    if (!c) return Q2D_EINVAL;
    const q2d_status s = check_cache_sizes(*c);
    if (s != Q2D_OK) return s;
    if (!c->k_codes || !c->v_codes_t || !c->k_scales || !c->v_scales || !on16(c->k_codes) || !on16(c->v_codes_t))
        return Q2D_EINVAL;
    return Q2D_OK;
}

// (a sequence's positions, sums of two of them and a tile's beyond its end stay within 32 bits)
q2d_status check_sequence_sizes(const q2d_kv_cache &c, const q2d_sequences *s)
{
    if (!s || s->batch <= 0 || s->tokens < 0 || s->table_pages <= 0 || s->table_stride < s->table_pages) return Q2D_EINVAL;
    if (!s->offsets && s->tokens % s->batch != 0) return Q2D_EINVAL;
    if (s->tokens > kMaxLen || s->batch > (1 << 20) || s->table_stride > kMaxLen) return Q2D_EUNSUPPORTED;
    if ((int64_t)s->table_pages * c.page_size > kMaxLen) return Q2D_EUNSUPPORTED;
    return Q2D_OK;
}

q2d_status check_sequences(const q2d_kv_cache &c, const q2d_sequences *s)
{
    const q2d_status r = check_sequence_sizes(c, s);
    if (r != Q2D_OK) return r;
    if (!s->lens || !s->table || !on4(s->lens) || !on4(s->table) || (reinterpret_cast<uintptr_t>(s->offsets) & 7) != 0)
        return Q2D_EINVAL;
    return Q2D_OK;
}

// [tokens][heads][dim] rows of whole 16 bytes
q2d_status check_rows(const void *p, int64_t tokens, int64_t st, int64_t heads, int64_t sh, int64_t dim, int per, bool output)
{
    const q2d_heads u = {const_cast<void *>(p), st, 0, sh};
    return output ? check_output(u, tokens, 1, heads, dim, per) : check_heads(u, tokens, 1, heads, dim, per);
}

Rows token_rows(const void *p, int64_t tokens, int64_t st, int64_t heads, int64_t sh, int64_t dim, int per)
{
    return rows_of({const_cast<void *>(p), st, 0, sh}, tokens, 1, heads, dim, per);
}

CacheView cache_view(const q2d_kv_cache *c)
{
    return {c->k_codes, c->v_codes_t, c->k_scales, c->v_scales, c->pages, c->heads, c->dim, c->page_size / 32};
}

SequencesView sequences_view(const q2d_sequences *s)
{
    return {s->offsets, s->lens, s->table, s->table_stride, s->table_pages, s->batch, s->tokens};
}

struct CachedSplit {
    int32_t units, wide;
    int64_t tiles, stat_at, bytes;
};

// Query tiles of 16 rows where the sequences have no more on average (decoding with up to 16
// query heads a key head), of 128 otherwise: a tile of 128 wastes what it does not fill, one of 16
// reads the cache again for each.  The rule looks at the call's average alone, and prompts take
// decoding sequences of the same call along: 60 of 600 to 8160 tokens and two prompts of 512
// take 222 us, in two calls 135 and 34 (two of 2048: 302, and 132 and 158).
// Sequences' tokens are cut into parts where the tiles alone would leave compute units short of
// four workgroups.  Four, though two run at once: 8 sequences of unequal length and work, 12644
// rows, take 384 us so and 428 us with two (4 equal ones of 64 new tokens each 82 and 70 us: the
// parts' way through memory, which equal work does not earn back).
CachedSplit split_cached(const q2d_kv_cache *c, const q2d_sequences *s, int32_t heads_q)
{
    CachedSplit p;
    const int64_t group = heads_q / c->heads;
    p.wide = s->tokens * group > 16 * (int64_t)s->batch;
    const int64_t rows = p.wide ? 128 : 16;
    if (s->offsets) {
        const int64_t some = s->tokens < s->batch ? s->tokens : s->batch, each = s->tokens * ((group + rows - 1) / rows);
        p.tiles = s->tokens * group / rows + some;
        if (each < p.tiles) p.tiles = each;
    } else {
        p.tiles = s->batch * ((s->tokens / s->batch * group + rows - 1) / rows);
    }
    // (never for tables that hold less than two parts)
    const int64_t longest = (int64_t)s->table_pages * c->page_size, least = p.wide ? 1024 : 512;
    const int64_t want = (4 * kComputeUnits + c->heads - 1) / c->heads;
    p.units = (int32_t)(p.tiles < want && longest >= least ? want : 0);
    const int64_t parts = p.units > 0 ? (p.tiles + p.units) * c->heads * rows : 0;
    p.stat_at = up256(parts * c->dim * 4);
    p.bytes = p.stat_at + up256(parts * 8);
    return p;
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
    const Rows q = query_rows(a, a->q), out = query_rows(a, a->out);
    if (!apart(out, key_rows(a, a->k)) || !apart(out, key_rows(a, a->v)) || !(same_rows(out, q) || apart(out, q)))
        return Q2D_EINVAL;
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
    // dK and dV are written before dQ's kernel reads q, k, v and dout; a workgroup of that writes
    // the rows whose q and dout it alone has read
    const Rows q = query_rows(a, a->q), k = key_rows(a, a->k), v = key_rows(a, a->v), g = query_rows(a, *dout);
    const Rows rq = query_rows(a, *dq), rk = key_rows(a, *dk), rv = key_rows(a, *dv);
    for (const Rows *x : {&rk, &rv})
        for (const Rows *y : {&q, &k, &v, &g, &rq})
            if (!apart(*x, *y)) return Q2D_EINVAL;
    if (!apart(rk, rv) || !apart(rq, k) || !apart(rq, v) || !(same_rows(rq, q) || apart(rq, q)) ||
        !(same_rows(rq, g) || apart(rq, g)))
        return Q2D_EINVAL;
    AttentionArgs r = make_args(a, workspace);
    r.dout = view(*dout); r.dq = view(*dq); r.dk = view(*dk); r.dv = view(*dv);
    if (launch_attention_bwd(r, a->dtype == Q2D_F32, stream) != hipSuccess) return Q2D_ELAUNCH;
    return Q2D_OK;
}

q2d_status q2d_kv_cache_init(q2d_kv_cache *c, int32_t pages, int32_t heads, int32_t dim, int32_t page_size,
                             int64_t bytes[4])
{
    if (!c) return Q2D_EINVAL;
    q2d_kv_cache t = {};
    t.pages = pages; t.heads = heads; t.dim = dim; t.page_size = page_size;
    const q2d_status s = check_cache_sizes(t);
    if (s != Q2D_OK) return s;
    *c = t;
    if (bytes) {
        const int64_t blocks = (int64_t)pages * heads * (page_size / 32);
        bytes[0] = bytes[1] = blocks * 32 * dim;
        bytes[2] = bytes[3] = blocks;
    }
    return Q2D_OK;
}

static q2d_status kv_copy(const q2d_kv_cache *c, const q2d_sequences *s, q2d_dtype dt, const void *k, int64_t kst,
                          int64_t ksh, const void *v, int64_t vst, int64_t vsh, bool write, hipStream_t stream)
{
    q2d_status r = check_cache(c);
    if (r == Q2D_OK) r = check_sequences(*c, s);
    if (r != Q2D_OK) return r;
    if (dt != Q2D_F32 && dt != Q2D_BF16) return Q2D_EINVAL;
    const int per = dt == Q2D_F32 ? 4 : 8;
    if (s->tokens == 0) return Q2D_OK;
    r = check_rows(k, s->tokens, kst, c->heads, ksh, c->dim, per, !write);
    if (r == Q2D_OK) r = check_rows(v, s->tokens, vst, c->heads, vsh, c->dim, per, !write);
    if (r != Q2D_OK) return r;
    if (!write && !apart(token_rows(k, s->tokens, kst, c->heads, ksh, c->dim, per),
                         token_rows(v, s->tokens, vst, c->heads, vsh, c->dim, per)))
        return Q2D_EINVAL;
    CacheCopyArgs a = {};
    a.cache = cache_view(c);
    a.seq = sequences_view(s);
    a.k = const_cast<void *>(k); a.k_st = kst; a.k_sh = ksh;
    a.v = const_cast<void *>(v); a.v_st = vst; a.v_sh = vsh;
    const hipError_t e = write ? launch_kv_write(a, dt == Q2D_F32, stream) : launch_kv_read(a, dt == Q2D_F32, stream);
    return e == hipSuccess ? Q2D_OK : Q2D_ELAUNCH;
}

q2d_status q2d_kv_write(const q2d_kv_cache *c, const q2d_sequences *s, q2d_dtype dt, const void *k, int64_t k_stride_token,
                        int64_t k_stride_head, const void *v, int64_t v_stride_token, int64_t v_stride_head,
                        hipStream_t stream)
{
    return kv_copy(c, s, dt, k, k_stride_token, k_stride_head, v, v_stride_token, v_stride_head, true, stream);
}

q2d_status q2d_kv_read(const q2d_kv_cache *c, const q2d_sequences *s, q2d_dtype dt, void *k, int64_t k_stride_token,
                       int64_t k_stride_head, void *v, int64_t v_stride_token, int64_t v_stride_head,
                       hipStream_t stream)
{
    return kv_copy(c, s, dt, k, k_stride_token, k_stride_head, v, v_stride_token, v_stride_head, false, stream);
}

int64_t q2d_attention_cached_workspace(const q2d_kv_cache *c, const q2d_sequences *s, int32_t heads_q)
{
    if (!c || !s || check_cache_sizes(*c) != Q2D_OK || check_sequence_sizes(*c, s) != Q2D_OK) return -1;
    if (heads_q <= 0 || heads_q % c->heads != 0) return -1;
    return split_cached(c, s, heads_q).bytes;
}

q2d_status q2d_attention_cached(const q2d_kv_cache *c, const q2d_sequences *s, const q2d_cached_attention *a,
                                void *workspace, int64_t workspace_bytes, hipStream_t stream)
{
    q2d_status r = check_cache(c);
    if (r == Q2D_OK) r = check_sequences(*c, s);
    if (r != Q2D_OK) return r;
    if (!a) return Q2D_EINVAL;
    if (a->dtype != Q2D_F32 && a->dtype != Q2D_BF16) return Q2D_EINVAL;
    if (a->dtype != Q2D_BF16) return Q2D_EUNSUPPORTED;
    if (a->heads_q <= 0 || a->heads_q % c->heads != 0 || a->window < 0) return Q2D_EINVAL;
    r = check_scale(a->scale, a->softcap);
    if (r != Q2D_OK) return r;
    if (!on4(a->slopes) || !on4(a->prefix)) return Q2D_EINVAL;
    if (s->tokens == 0) return Q2D_OK;
    if (s->tokens > INT32_MAX / a->heads_q) return Q2D_EUNSUPPORTED;
    r = check_rows(a->q, s->tokens, a->q_stride_token, a->heads_q, a->q_stride_head, c->dim, 8, false);
    if (r == Q2D_OK) r = check_rows(a->out, s->tokens, a->out_stride_token, a->heads_q, a->out_stride_head, c->dim, 8, true);
    if (r != Q2D_OK) return r;
    const CachedSplit p = split_cached(c, s, a->heads_q);
    r = check_workspace(p.bytes, workspace, workspace_bytes);
    if (r != Q2D_OK) return r;
    const Rows rows = token_rows(a->q, s->tokens, a->q_stride_token, a->heads_q, a->q_stride_head, c->dim, 8);
    const Rows out = token_rows(a->out, s->tokens, a->out_stride_token, a->heads_q, a->out_stride_head, c->dim, 8);
    if (!same_rows(out, rows) && !apart(out, rows)) return Q2D_EINVAL;
    CachedArgs g = {};
    g.cache = cache_view(c);
    g.seq = sequences_view(s);
    g.q = a->q; g.q_st = a->q_stride_token; g.q_sh = a->q_stride_head;
    g.out = a->out; g.out_st = a->out_stride_token; g.out_sh = a->out_stride_head;
    g.mask.causal = 1;
    g.mask.window = (int32_t)(a->window > kMaxLen ? kMaxLen : a->window);
    g.mask.scale = a->scale; g.mask.cap = a->softcap;
    g.mask.slopes = a->slopes; g.mask.prefix = a->prefix;
    g.heads_q = a->heads_q;
    g.units = p.units; g.wide = p.wide; g.tiles = p.tiles;
    g.part = reinterpret_cast<float *>(workspace);
    g.stat = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(workspace) + p.stat_at);
    if (launch_attention_cached(g, stream) != hipSuccess) return Q2D_ELAUNCH;
    return Q2D_OK;
}

}  // extern "C"
