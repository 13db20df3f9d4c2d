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
    int2 *ranges;                    // [batch][ceil(len_k / 64)] document ranges (workspace)
    AttentionMask mask;
    int32_t batch, len_q, len_k, heads_q, heads_kv, dim;
};

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
    int32_t splits;                              // parts of a sequence's tokens
    int32_t wide;                                // 64 query rows a workgroup, not 16
    int64_t tiles;                               // bound of the query tiles of all sequences
    float *part;                                 // workspace: [tile][head][split][rows][dim] sums,
    float *stat;                                 // [tile][head][split][rows] maximum and sum
};

hipError_t launch_kv_write(const CacheCopyArgs &a, bool f32, hipStream_t stream);
hipError_t launch_kv_read(const CacheCopyArgs &a, bool f32, hipStream_t stream);
hipError_t launch_attention_cached(const CachedArgs &a, hipStream_t stream);

}  // namespace q2d
