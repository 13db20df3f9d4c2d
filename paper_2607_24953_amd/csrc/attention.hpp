// Launch interface of the attention and cache kernels (host and device side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace q2d {

// Which pairs are seen, and how their scores are changed
struct AttentionMask {
    int32_t causal;
    int32_t window;                  // 0: none
    float scale, cap;                // cap 0: none
    const float *slopes;             // [heads_q], or null
    const int32_t *documents;        // [batch][len_k], or null
    const int32_t *prefix;           // [batch], or null
};

// [batch][length][heads][dim], strides in elements, unit stride along dim
struct HeadsView {
    void *p;
    int64_t sb, sl, sh;
};

struct AttentionArgs {
    HeadsView q, k, v, out;
    HeadsView dout, dq, dk, dv;      // backward
    float *lse;                      // [batch][heads_q][len_q], natural logarithm
    float *delta, *lse2;             // [batch][heads_q][len_q], backward workspace: delta, lse log2 e
    float *part;                     // [2][splits][batch][len_k][heads_kv][dim] sums of dK and dV (workspace)
    int2 *ranges;                    // [batch][ceil(len_k / 64)] document ranges (workspace)
    AttentionMask mask;
    int32_t batch, len_q, len_k, heads_q, heads_kv, dim;
    int32_t splits;                  // backward: parts of the query heads that share a key head
};

constexpr int kComputeUnits = 256;

// What a kernel does to scores, its template argument MODS: bit 0 caps them, bit 1 adds the
// distance bias, bit 2 (bfloat16, in kAnyCap alone) takes caps of any size.
//
// Caps up to kNarrowCap (the usual ones are 20 to 50) take tanh with an error of 2^-23 of 1, scores
// then with one of 2^-23 of the cap: below 2^-17, far below the bf16 operands' rounding.  That
// error would grow with the cap (weights off by a factor of 2 at 10^7), so those above take
// tanh with a small relative error, for ten instructions more a score: 2 x 4096 tokens, 16 heads
// of 128 dims, forward 325 us in place of 260, backward 917 in place of 746.  One kernel does so,
// with a bias whose slopes may be 0.
constexpr float kNarrowCap = 64.f;
constexpr int kAnyCap = 7;

inline int mods_of(const AttentionMask &m, bool f32)
{
    if (m.cap > kNarrowCap && !f32) return kAnyCap;
    return (m.cap > 0.f ? 1 : 0) | (m.slopes ? 2 : 0);
}

// Parts that the query heads sharing a key head are cut into for dK and dV, each summed by
// workgroups (of 128 keys) of its own and then joined from float32 in memory.  Where there are
// fewer than four workgroups a compute unit, as many parts as bring them there: 1 x 4096
// tokens, 32 on 8 heads, 128 dims, backward 844 -> 684 us with 4.  With documents, whose
// workgroups differ in work, 16 a compute unit in place of 4: 16384 tokens, 32 on 8 heads, 64 dims,
// 1611 -> 1332 us; 4 x 4096 tokens 1339 -> 1124, with 128 dims 1941 -> 1838; 8192 tokens, 32 on 4
// heads, 128 dims 1310 -> 1252; 2 x 2048 tokens, 16 on 4 heads, 64 dims 195 and 194.  But not so
// many that writing and reading the parts outweighs it, a part a thousand (from one workgroup a
// compute unit on, four thousand) rows of queries at most: 4 x 1024 tokens of the first case are
// 269 us with 1 part and 306 with 4.
inline int dkv_splits(int64_t batch, int64_t len_q, int64_t len_k, int heads_q, int heads_kv, bool documents)
{
    const int64_t n = batch * heads_kv * ((len_k + 127) / 128), group = heads_q / heads_kv;
    int64_t parts = ((documents ? 16 : 4) * kComputeUnits + n - 1) / n;
    const int64_t most = len_q * group / (n < kComputeUnits ? 1024 : 4096);
    if (parts > most) parts = most;
    if (parts > group) parts = group;
    if (parts < 1) parts = 1;
    const int64_t each = (group + parts - 1) / parts;
    return (int)((group + each - 1) / each);
}

// fills a.ranges
hipError_t launch_document_ranges(const AttentionArgs &a, hipStream_t stream);
hipError_t launch_attention_fwd(const AttentionArgs &a, bool f32, hipStream_t stream);
hipError_t launch_attention_bwd(const AttentionArgs &a, bool f32, hipStream_t stream);

// A paged cache of E4M3 keys and values: one scale byte for each block of 32 tokens and
// head; keys [page][head][token][dim], values transposed in their block
// [page][head][block][dim][32].
struct CacheView {
    uint8_t *k, *v, *ks, *vs;
    int32_t pages, heads, dim, page_blocks;      // blocks of 32 tokens a page
};

// Sequences whose last n[b] = offsets[b + 1] - offsets[b] tokens a call works on (offsets
// null: tokens / batch each); lens[b]: tokens of the sequence, table[b][i]: its pages
struct SequencesView {
    const int64_t *offsets;
    const int32_t *lens, *table;
    int64_t table_stride;
    int32_t table_pages, batch;
    int64_t tokens;
};

struct CacheCopyArgs {
    CacheView cache;
    SequencesView seq;
    void *k, *v;
    int64_t k_st, k_sh, v_st, v_sh;              // strides of tokens and heads, elements
};

struct CachedArgs {
    CacheView cache;
    SequencesView seq;
    const void *q;
    void *out;
    int64_t q_st, q_sh, out_st, out_sh;
    AttentionMask mask;
    int32_t heads_q;
    int32_t units;                               // work units a head to cut long sequences for, 0: do not
    int32_t wide;                                // 128 query rows a workgroup, not 16
    int32_t grid;                                // workgroups of the units; those past them clear (zero_rows)
    int64_t tiles;                               // bound of the query tiles of all sequences
    float *part;                                 // workspace: [unit][head][rows][dim] sums,
    float *stat;                                 // [unit][head][rows] maximum and sum
};

constexpr int kMaxSplits = 64;                   // parts of a sequence's tokens: a lane each in the join

hipError_t launch_kv_write(const CacheCopyArgs &a, bool f32, hipStream_t stream);
hipError_t launch_kv_read(const CacheCopyArgs &a, bool f32, hipStream_t stream);
hipError_t launch_attention_cached(const CachedArgs &a, hipStream_t stream);

}  // namespace q2d
