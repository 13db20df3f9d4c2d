// Writing new tokens into the paged 8-bit cache, and reading tokens back as values.
//
// Both are memory-bound: 16384 tokens of 32 heads and 128 dims, bfloat16, keys and values, are
// written (403 MB read and written) in 100 to 109 us, 3.7 to 4 TB/s, and read back in 71 to 84 us,
// 4.8 to 5.7 TB/s, where a large copy reaches 4.9.  One token of each of 64 sequences takes 7 and 6 us, a launch and
// the chain offsets, page table, block.  The write gains nothing from more bytes under way: a
// lane's 8 rows are loaded at once, and the scale needs all of them.
//
// A wave takes one block of 32 tokens of one head, keys or values:
// lane (tg, dg) holds the 8 x 8 elements of tokens 8 tg .. and dims 8 dg .., loaded as 16 or
// 32 bytes a token.  The E4M3 codes come from v_cvt_scalef32_pk_fp8_f32, pairs along dims for
// keys and along tokens for the transposed values, so that both leave in 8-byte stores with
// no exchange between lanes.
#include "cache_common.hpp"

namespace q2d {

namespace {

typedef short s2v __attribute__((ext_vector_type(2)));

// E4M3 codes (to nearest even) of four values over a power-of-two scale
__device__ __forceinline__ uint32_t fp8_quad(float a, float b, float c, float d, float scale)
{
    s2v r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
    return __builtin_bit_cast(uint32_t, r);
}

// four values of E4M3 codes times 2^(byte - 127); a scale byte of 255 is a NaN
__device__ __forceinline__ void fp8_values(uint32_t codes, uint32_t byte, float *x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float v = ldexpf(__builtin_amdgcn_cvt_f32_fp8((int)codes >> (8 * i), 0), (int)byte - 127);
        x[i] = byte == 255 ? __builtin_nanf("") : v;
    }
}

template <typename T>
__device__ __forceinline__ void load8(const T *p, float *x)
{
    if constexpr (sizeof(T) == 4) {
        const v4f a = *reinterpret_cast<const v4f *>(p), b = *reinterpret_cast<const v4f *>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
    } else {
        const u4v v = *reinterpret_cast<const u4v *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = bits_f(v[i] << 16); x[2 * i + 1] = bits_f(v[i] & 0xFFFF0000u); }
    }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, const float *x)
{
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<v4f *>(p) = v4f{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<v4f *>(p + 4) = v4f{x[4], x[5], x[6], x[7]};
    } else {
        typedef __bf16 b8 __attribute__((ext_vector_type(8)));
        b8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
        *reinterpret_cast<b8 *>(p) = v;
    }
}

// the blocks that the last n of len tokens lie in (tokens before the first position are left out)
__device__ __forceinline__ int touched(const Span &s)
{
    const int n = min(s.n, s.len);
    return n == 0 ? 0 : (s.len + kBlockTokens - 1) / kBlockTokens - (s.len - n) / kBlockTokens;
}

// One wave's work: block `block` of sequence b (at: its number, -1 on no page), slots [lo, hi)
// of it, rows `row0` + slot
struct Unit {
    int64_t at, row0;
    int lo, hi, head;
    bool values;
};

__device__ __forceinline__ bool take_unit(const CacheCopyArgs &a, Unit &u)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // neighbouring workgroups take the heads of one block: a token's heads lie side by side
    const uint32_t parts = (2 * a.cache.heads + 3) / 4;
    const int part = blockIdx.x % parts * 4 + wave;
    if (part >= 2 * a.cache.heads) return false;
    Span s;
    int i;
    const int b = find_unit(a.seq, a.cache.page_blocks * kBlockTokens, blockIdx.x / parts, touched, s, i);
    if (b < 0) return false;
    const int n = min(s.n, s.len), first = s.len - n, block = first / kBlockTokens + i;
    u.head = part >> 1;
    u.values = part & 1;
    u.lo = max(first - block * kBlockTokens, 0);
    u.hi = min(s.len - block * kBlockTokens, kBlockTokens);
    u.row0 = s.tok0 + (s.n - n) + (int64_t)block * kBlockTokens - first;
    u.at = cache_block(a.cache, a.seq, b, block, u.head);
    return true;
}

template <typename T>
__global__ __launch_bounds__(256) void kv_write_kernel(const CacheCopyArgs a)
{
    Unit u;
    if (!take_unit(a, u) || u.at < 0) return;
    const int lane = threadIdx.x & 63, tg = lane >> 4, dg = lane & 15, D = a.cache.dim, s0 = 8 * tg;
    const bool on = 8 * dg < D;
    const T *x = (const T *)(u.values ? a.v : a.k) + u.head * (u.values ? a.v_sh : a.k_sh) + 8 * dg;
    const int64_t st = u.values ? a.v_st : a.k_st;
    float e[8][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[i][j] = 0.f;
        if (on && s0 + i >= u.lo && s0 + i < u.hi) load8(x + (u.row0 + s0 + i) * st, e[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, f_bits(e[i][j]) & 0x7FFFFFFFu);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    uint32_t byte = top >= 0x7F800000u ? 255u : (uint32_t)(fp8_block_exponent(top) + 127);
    uint8_t *scale_at = (u.values ? a.cache.vs : a.cache.ks) + u.at;
    const uint32_t before = u.lo > 0 ? *scale_at : byte;
    // The scale of tokens already there only grows; their codes are then rounded to the new one
    // (to nearest even, a second rounding: the values they came from are gone)
    byte = max(byte, before);
    const bool redo = u.lo > 0 && byte != before;
    const float scale = bits_f((byte == 255 ? 127u : byte) << 23);
    const int64_t base = u.at * kBlockTokens * D;
    if (!on) {
    } else if (!u.values) {
        uint8_t *p = a.cache.k + base + 8 * dg;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int s = s0 + i;
            if (s >= u.hi || (s < u.lo && !redo)) continue;
            if (s < u.lo) {
                const uint2 w = *reinterpret_cast<const uint2 *>(p + (int64_t)s * D);
                fp8_values(w.x, before, e[i]);
                fp8_values(w.y, before, e[i] + 4);
            }
            uint2 w = make_uint2(fp8_quad(e[i][0], e[i][1], e[i][2], e[i][3], scale),
                                 fp8_quad(e[i][4], e[i][5], e[i][6], e[i][7], scale));
            if (byte == 255) w = make_uint2(0, 0);
            *reinterpret_cast<uint2 *>(p + (int64_t)s * D) = w;
        }
    } else {
        uint8_t *p = a.cache.v + base + (int64_t)8 * dg * kBlockTokens + s0;
        // bytes of this lane's 8 slots that hold earlier tokens
        const int nk = min(max(u.lo - s0, 0), 8);
        const uint64_t kept = nk == 8 ? ~0ull : (1ull << (8 * nk)) - 1;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint64_t old = 0;
            if (nk > 0) {
                old = *reinterpret_cast<const uint64_t *>(p + j * kBlockTokens);
                if (redo) {
                    float y[8];
                    fp8_values((uint32_t)old, before, y);
                    fp8_values((uint32_t)(old >> 32), before, y + 4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i][j] = i < nk ? y[i] : e[i][j];
                }
            }
            const uint64_t lo = fp8_quad(e[0][j], e[1][j], e[2][j], e[3][j], scale);
            const uint64_t hi = fp8_quad(e[4][j], e[5][j], e[6][j], e[7][j], scale);
            uint64_t w = lo | (hi << 32);
            if (!redo) w = (w & ~kept) | (old & kept);
            if (byte == 255) w = 0;
            *reinterpret_cast<uint64_t *>(p + j * kBlockTokens) = w;
        }
    }
    if (lane == 0) *scale_at = (uint8_t)byte;
}

// Rows that no token stands behind are zeros: those of no sequence, and a sequence's before its
// first position
template <typename T>
__device__ __forceinline__ void clear_rows(const CacheCopyArgs &a, int group, int groups)
{
    T *k = (T *)a.k, *v = (T *)a.v;
    auto clear = [&](int64_t row, int64_t n, int64_t first, int64_t step) {
        zero_rows(k + row * a.k_st, a.k_st, a.k_sh, n, a.cache.heads, a.cache.dim, first, step);
        zero_rows(v + row * a.v_st, a.v_st, a.v_sh, n, a.cache.heads, a.cache.dim, first, step);
    };
    const int64_t thread = group * 256 + threadIdx.x, threads = groups * 256;
    const Outside x = outside_of(a.seq);
    clear(0, x.lo, thread, threads);
    clear(x.hi, a.seq.tokens - x.hi, thread, threads);
    const int lane = threadIdx.x & 63;
    for (int64_t base = thread - lane; base < a.seq.batch; base += threads) {
        Span s = {0, 0, 0};
        if (base + lane < a.seq.batch) s = span_of(a.seq, a.cache.page_blocks * kBlockTokens, (int)base + lane);
        for (uint64_t some = __ballot(s.n > s.len); some; some &= some - 1) {
            const int at = __builtin_ctzll(some);
            clear(__shfl(s.tok0, at), __shfl(s.n - s.len, at), lane, 64);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void kv_read_kernel(const CacheCopyArgs a, int grid)
{
    if (blockIdx.x >= (uint32_t)grid) return clear_rows<T>(a, blockIdx.x - grid, gridDim.x - grid);
    Unit u;
    if (!take_unit(a, u)) return;
    const int lane = threadIdx.x & 63, tg = lane >> 4, dg = lane & 15, D = a.cache.dim, s0 = 8 * tg;
    if (8 * dg >= D) return;
    T *x = (T *)(u.values ? a.v : a.k) + u.head * (u.values ? a.v_sh : a.k_sh) + 8 * dg;
    const int64_t st = u.values ? a.v_st : a.k_st, base = u.at * kBlockTokens * D;
    if (u.at < 0) {
        const float none[8] = {};
        for (int s = max(s0, u.lo); s < min(s0 + 8, u.hi); ++s) store8(x + (u.row0 + s) * st, none);
        return;
    }
    float e[8][8];
    const uint32_t byte = *((u.values ? a.cache.vs : a.cache.ks) + u.at);
    if (!u.values) {
        const uint8_t *p = a.cache.k + base + 8 * dg;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint2 w = *reinterpret_cast<const uint2 *>(p + (int64_t)(s0 + i) * D);
            fp8_values(w.x, byte, e[i]);
            fp8_values(w.y, byte, e[i] + 4);
        }
    } else {
        const uint8_t *p = a.cache.v + base + (int64_t)8 * dg * kBlockTokens + s0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint2 w = *reinterpret_cast<const uint2 *>(p + j * kBlockTokens);
            float y[8];
            fp8_values(w.x, byte, y);
            fp8_values(w.y, byte, y + 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i][j] = y[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (s0 + i >= u.lo && s0 + i < u.hi) store8(x + (u.row0 + s0 + i) * st, e[i]);
}

// workgroups: a sequence's n tokens lie in at most (n + 30) / 32 + 1 blocks
int64_t grid_of(const CacheCopyArgs &a)
{
    int64_t blocks;
    if (a.seq.offsets) {
        const int64_t some = a.seq.tokens < a.seq.batch ? a.seq.tokens : a.seq.batch;
        blocks = (a.seq.tokens + 30 * some) / kBlockTokens + some;
        blocks = blocks < a.seq.tokens ? blocks : a.seq.tokens;
    } else {
        const int64_t n = a.seq.tokens / a.seq.batch;
        blocks = n == 0 ? 0 : a.seq.batch * ((n + 30) / kBlockTokens + 1);
    }
    return blocks * ((2 * a.cache.heads + 3) / 4);
}

}  // namespace

hipError_t launch_kv_write(const CacheCopyArgs &a, bool f32, hipStream_t stream)
{
    const int64_t grid = grid_of(a);
    if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
    if (grid == 0) return hipSuccess;
    if (f32) kv_write_kernel<float><<<(uint32_t)grid, 256, 0, stream>>>(a);
    else kv_write_kernel<__bf16><<<(uint32_t)grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv_read(const CacheCopyArgs &a, bool f32, hipStream_t stream)
{
    const int64_t grid = grid_of(a);
    const uint32_t all = (uint32_t)grid + zero_groups(a.seq.tokens > a.seq.batch ? a.seq.tokens : a.seq.batch);
    if (grid > INT32_MAX - 256) return hipErrorInvalidConfiguration;
    if (grid == 0) return hipSuccess;
    if (f32) kv_read_kernel<float><<<all, 256, 0, stream>>>(a, (int)grid);
    else kv_read_kernel<__bf16><<<all, 256, 0, stream>>>(a, (int)grid);
    return hipGetLastError();
}

}  // namespace q2d
