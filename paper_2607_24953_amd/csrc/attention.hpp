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
    float *delta;                    // [batch][heads_q][len_q], backward workspace
    int2 *ranges;                    // [batch][ceil(len_k / 64)] document ranges (workspace)
    AttentionMask mask;
    int32_t batch, len_q, len_k, heads_q, heads_kv, dim;
};

// fills a.ranges
hipError_t launch_document_ranges(const AttentionArgs &a, hipStream_t stream);
hipError_t launch_attention_fwd(const AttentionArgs &a, bool f32, hipStream_t stream);
hipError_t launch_attention_bwd(const AttentionArgs &a, bool f32, hipStream_t stream);

}  // namespace q2d
