// Device helpers of the kernels on the paged 8-bit cache.
#pragma once

#include "attention.hpp"
#include "device_common.hpp"

namespace q2d {
namespace {

constexpr int kBlockTokens = 32;

// Tokens that a call works on in one sequence: positions [len - n, len), rows tok0 .. of
// the token tensors.  Offsets and lengths come from the device unchecked: clamped to the
// token tensors and to what the page table can hold.
struct Span {
    int n, len;
    int64_t tok0;
};

__device__ __forceinline__ Span span_of(const SequencesView &s, int page_tokens, int b)
{
    Span r;
    if (s.offsets) {
        const int64_t lo = min(max(s.offsets[b], (int64_t)0), s.tokens);
        const int64_t hi = min(max(s.offsets[b + 1], lo), s.tokens);
        r.tok0 = lo;
        r.n = (int)(hi - lo);
    } else {
        r.n = (int)(s.tokens / s.batch);
        r.tok0 = (int64_t)b * r.n;
    }
    r.len = (int)min((int64_t)max(s.lens[b], 0), (int64_t)s.table_pages * page_tokens);
    return r;
}

// Rows of the token tensors that belong to no sequence: [0, lo) and [hi, tokens)
struct Outside { int64_t lo, hi; };

__device__ __forceinline__ Outside outside_of(const SequencesView &s)
{
    Outside r = {0, s.tokens};
    if (s.offsets) {
        r.lo = min(max(s.offsets[0], (int64_t)0), s.tokens);
        r.hi = min(max(s.offsets[s.batch], r.lo), s.tokens);
    }
    return r;
}

// Zeros in n rows [heads][dim] from x on (strides in elements), by threads first, first + step, ..
template <typename T>
__device__ __forceinline__ void zero_rows(T *x, int64_t st, int64_t sh, int64_t n, int heads, int dim, int64_t first, int64_t step)
{
    const int chunks = dim * (int)sizeof(T) / 16, row = heads * chunks;
    for (int64_t i = first; i < n * row; i += step) {
        const int64_t r = i / row;
        const int c = (int)(i % row);
        *reinterpret_cast<u4v *>(x + r * st + c / chunks * sh + c % chunks * (16 / (int)sizeof(T))) = u4v{0, 0, 0, 0};
    }
}

// workgroups that do so beside a call's own: a call that leaves no such rows has them look once
inline int zero_groups(int64_t tokens) { return tokens < 256 ? 1 : tokens > 65536 ? 256 : (int)(tokens / 256); }

// Unit `index` of all sequences' units, sequence b having count(span) of them: its
// sequence, its number there and the span; b = -1 past the last.  One full wave, the same
// answer in all lanes.
template <typename F>
__device__ __forceinline__ int find_unit(const SequencesView &s, int page_tokens, int64_t index, F &&count, Span &span, int &unit)
{
    const int lane = threadIdx.x & 63;
    int64_t carry = 0;
    for (int base = 0; base < s.batch; base += 64) {
        const int b = base + lane;
        Span mine = {0, 0, 0};
        int c = 0;
        if (b < s.batch) {
            mine = span_of(s, page_tokens, b);
            c = count(mine);
        }
        int64_t upto = c;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t below = __shfl_up(upto, d);
            if (lane >= d) upto += below;
        }
        const uint64_t past = __ballot(carry + upto > index);
        if (past) {
            const int at = __builtin_ctzll(past);
            span.n = __builtin_amdgcn_readlane(mine.n, at);
            span.len = __builtin_amdgcn_readlane(mine.len, at);
            const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)mine.tok0, at);
            const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)mine.tok0 >> 32), at);
            span.tok0 = (int64_t)(((uint64_t)hi << 32) | lo);
            const int64_t first = carry + __shfl(upto, at) - __shfl(c, at);
            unit = __builtin_amdgcn_readfirstlane((int)(index - first));
            return base + at;
        }
        carry += __shfl(upto, 63);
    }
    return -1;
}

// Block number of (page, head, block of the page) in scale arrays; -1 where the table
// names no page of the cache
__device__ __forceinline__ int64_t cache_block(const CacheView &c, const SequencesView &s, int b, int block, int head)
{
    const int page = s.table[(int64_t)b * s.table_stride + block / c.page_blocks];
    if ((uint32_t)page >= (uint32_t)c.pages) return -1;
    return ((int64_t)page * c.heads + head) * c.page_blocks + block % c.page_blocks;
}

}  // namespace
}  // namespace q2d
