// Device helpers of the attention kernels: operand fragments on the matrix cores, LDS
// tiles, and the masks.
//
// Every product runs as D[m][n] += A[m][k] B[k][n] on 32 x 32 output tiles with k in
// steps of 16, and the kernels choose which operand is A so that a softmax row lies in
// one lane pair: lane l holds column n = l % 32 and the 16 rows 8 (i / 4) + 4 (l / 32) +
// i % 4.  A fragment gives lane l row (or column) l % 32 and 8 values of k, which may be
// any 8 as long as A and B agree.  So an output tile turned into the B operand of the
// next product needs no exchange between lanes: its registers 8 s .. 8 s + 7 are k-step
// s, for an A fragment that holds the same rows (column_frag).
//
// float32 operands take eight v_mfma_f32_32x32x2_f32 a step on the same fragments.
#pragma once

#include <math.h>
#include "attention.hpp"
#include "gemm_common.hpp"

namespace q2d {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v8f __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <typename T> struct FragOf;
template <> struct FragOf<__bf16> { typedef bf16x8 type; };
template <> struct FragOf<float> { typedef v8f type; };
template <typename T> using Frag = typename FragOf<T>::type;

__device__ __forceinline__ v16f mma(bf16x8 a, bf16x8 b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ v16f mma(v8f a, v8f b, v16f c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

// registers 8 s .. 8 s + 7 of an output tile as an operand fragment (bf16: to nearest even)
template <typename T>
__device__ __forceinline__ Frag<T> to_frag(const v16f &x, int s)
{
    Frag<T> f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = x[8 * s + j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const v2f v = {x[8 * s + j], x[8 * s + j + 1]};
            const bf16x2v w = __builtin_convertvector(v, bf16x2v);
            f[j] = w[0];
            f[j + 1] = w[1];
        }
    }
    return f;
}

// An LDS tile of rows of DT elements of T, in 16-byte chunks whose place in a row is
// XORed with a function of the row number: neighbouring rows then start on different
// banks, for reads along rows (row_frag: 16 bytes each of up to 32 rows) and across
// them (column_frag: 32 or 64 bytes of 4 neighbouring rows).
template <typename T, int DT>
struct Tile {
    static constexpr int kPer = 16 / sizeof(T);            // elements a chunk
    static constexpr int kChunks = DT / kPer;              // chunks a row
    static constexpr int kRowBytes = DT * sizeof(T);

    static __device__ __forceinline__ int swizzle(int r)
    {
        if constexpr (sizeof(T) == 4) return r & (kChunks == 32 ? 7 : 15);
        else if constexpr (kChunks == 16) return ((r & 3) << 2) | ((r >> 2) & 3);
        else return ((r & 2) << 1) | ((r >> 2) & 3);
    }
    static __device__ __forceinline__ int offset(int r, int chunk) { return r * kRowBytes + ((chunk ^ swizzle(r)) << 4); }

    // LDS address of a tile for the reads below, per lane.  The kernels form it anew for each
    // tile (fresh): the addresses of the reads are then sums and XORs with constants at the
    // read, in place of dozens of registers kept over the loop.
    static __device__ __forceinline__ uint32_t address(const uint8_t *t)
    {
        return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t *)t;
    }
    // of row lane % 32, for row_frag
    static __device__ __forceinline__ uint32_t row_base(const uint8_t *t, int lane)
    {
        const int r = lane & 31, h = lane >> 5;
        return fresh(address(t) + offset(r, sizeof(T) == 2 ? h : 2 * h));
    }
    // for column_frag
    static __device__ __forceinline__ uint32_t column_base(const uint8_t *t, int lane)
    {
        const int h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            // ds_read_b64_tr_b16 hands lane i of each 16 the i-th column of a 4 x 16 block
            // whose rows the lanes 4 r .. 4 r + 3 point at
            const int i = lane & 15, r = 4 * h + (i >> 2);
            const int chunk = 2 * ((lane >> 4) & 1) + ((i >> 1) & 1), half = (i & 1) << 3;
            return fresh(address(t) + offset(r, chunk) + half);
        } else {
            const int d = lane & 31;
            return fresh(address(t) + offset(4 * h, d >> 2) + ((d & 3) << 2));
        }
    }
    static __device__ __forceinline__ uint32_t fresh(uint32_t a)
    {
        asm("" : "+v"(a));
        return a;
    }

    // 8 elements 16 ks + 8 h .. (h = lane / 32) of row 32 t + lane % 32; tiles are aligned to
    // kRowBytes, and swizzle(r + 32) == swizzle(r), so that a chunk number's bits are XORed in
    static __device__ __forceinline__ Frag<T> row_frag(uint32_t base, int t, int ks)
    {
        if constexpr (sizeof(T) == 2) {
            return *lds_ptr<bf16x8>((base ^ (uint32_t)(ks << 5)) + 32 * t * kRowBytes);
        } else {
            const v4f a = *lds_ptr<v4f>((base ^ (uint32_t)(ks << 6)) + 32 * t * kRowBytes);
            const v4f b = *lds_ptr<v4f>((base ^ (uint32_t)((ks << 6) | 16)) + 32 * t * kRowBytes);
            return v8f{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        }
    }

    // column 32 dt + lane % 32, rows r0 + 4 h + 0..3 and r0 + 8 + 4 h + 0..3, r0 a multiple of 16
    static __device__ __forceinline__ Frag<T> column_frag(uint32_t base, int r0, int dt)
    {
        if constexpr (sizeof(T) == 2) {
            typedef __attribute__((address_space(3))) v4s *lp;
            // (swizzle(r + 8) differs from swizzle(r) in bit 1)
            const uint32_t x = base ^ (uint32_t)(dt << 6);
            const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(uintptr_t)(x + r0 * kRowBytes));
            const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(uintptr_t)((x ^ 32u) + (r0 + 8) * kRowBytes));
            const bf16x4 u = __builtin_bit_cast(bf16x4, a), v = __builtin_bit_cast(bf16x4, b);
            return __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            v8f f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = r0 + (j & 3) + 2 * (j & 4);              // + 4 h in the base: swizzle's bits 0, 1 and 3
                const uint32_t x = base ^ (uint32_t)((swizzle(r) << 4) ^ (dt << 7));
                f[j] = *lds_ptr<float>(x + r * kRowBytes);
            }
            return f;
        }
    }
    template <typename V>
    static __device__ __forceinline__ const __attribute__((address_space(3))) V *lds_ptr(uint32_t a)
    {
        return (const __attribute__((address_space(3))) V *)(uintptr_t)a;
    }

    // Fills ROWS rows from row r0 of a matrix of n rows (base; stride in elements, below
    // 2^22) and D columns with NT threads, asynchronously (wait_vmcnt).  Rows from n on
    // repeat row n - 1; columns from D on keep what the tile holds (clear).
    template <int ROWS, int NT>
    static __device__ __forceinline__ void load(uint8_t *t, const T *base, int64_t stride, int r0, int n, int D)
    {
        constexpr int RP = NT / kChunks;                       // rows a pass; swizzle(r + RP) == swizzle(r)
        static_assert(ROWS % RP == 0 && (RP % 16 == 0 || (RP % 8 == 0 && kChunks == 32)), "whole passes");
        const int tid = threadIdx.x, r = tid / kChunks;
        const int d = ((tid % kChunks) ^ swizzle(r)) * kPer;
        const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t *)t +
                             __builtin_amdgcn_readfirstlane(tid & ~63) * 16;
        const uint32_t pitch = (uint32_t)stride * sizeof(T);
        const uint8_t *src = reinterpret_cast<const uint8_t *>(base + (int64_t)r0 * stride);
        if (d >= D) return;
        if (r0 + ROWS <= n) {
            const uint32_t off = r * pitch + d * sizeof(T);
#pragma unroll
            for (int i = 0; i < ROWS / RP; ++i)
                lds_dma16(src + (uint64_t)(i * RP) * pitch, off, lds + i * NT * 16);
        } else {
#pragma unroll
            for (int i = 0; i < ROWS / RP; ++i)
                lds_dma16(src, (uint32_t)min(r + i * RP, n - 1 - r0) * pitch + d * sizeof(T), lds + i * NT * 16);
        }
    }

    // zeros in `bytes` bytes of tiles, for the columns from D on
    template <int NT>
    static __device__ __forceinline__ void clear(uint8_t *t, int bytes)
    {
        for (int i = threadIdx.x * 16; i < bytes; i += NT * 16) *reinterpret_cast<u4v *>(t + i) = u4v{0, 0, 0, 0};
    }

    static __device__ __forceinline__ bool chunk_non_finite(u4v v)
    {
        bool bad = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 4) bad |= (v[j] & 0x7f800000u) == 0x7f800000u;
            else bad |= (v[j] & 0x7f80u) == 0x7f80u || (v[j] & 0x7f800000u) == 0x7f800000u;
        }
        return bad;
    }

    // zeros in place of infinities and NaN, by all threads; barriers before and after
    template <int ROWS, int NT>
    static __device__ __forceinline__ void clean(uint8_t *t)
    {
        wait_lgkm();
        block_barrier();
#pragma unroll 1
        for (int i = threadIdx.x; i < ROWS * kChunks; i += NT) {
            u4v v = *reinterpret_cast<const u4v *>(t + i * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 4) {
                    v[j] = (v[j] & 0x7f800000u) == 0x7f800000u ? 0u : v[j];
                } else {
                    v[j] = (v[j] & 0x7f80u) == 0x7f80u ? v[j] & 0xffff0000u : v[j];
                    v[j] = (v[j] & 0x7f800000u) == 0x7f800000u ? v[j] & 0xffffu : v[j];
                }
            }
            *reinterpret_cast<u4v *>(t + i * 16) = v;
        }
        wait_lgkm();
        block_barrier();
    }
};

// 64 neighbouring 32-bit numbers from base[i0] to LDS, by one wave; indices clamped to [0, n)
__device__ __forceinline__ void load_words64(void *lds, const void *base, int i0, int n)
{
    const int i = min(max(i0 + (int)(threadIdx.x & 63), 0), n - 1);
    lds_dma4(reinterpret_cast<const uint8_t *>(base) + (int64_t)i * 4,
             __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds));
}

// row of an output tile that register i of lane half h holds
__device__ __forceinline__ int tile_row(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// One 8-element operand fragment of a matrix row straight from memory: elements
// 16 ks + 8 h ..; zeros where the row or the columns lie outside
template <typename T>
__device__ __forceinline__ Frag<T> global_frag(const T *row, bool valid, int ks, int h, int D)
{
    const int d = 16 * ks + 8 * h;
    Frag<T> f = {};
    if (valid && d < D) {
        if constexpr (sizeof(T) == 2) {
            f = *reinterpret_cast<const bf16x8 *>(row + d);
        } else {
            const v4f a = *reinterpret_cast<const v4f *>(row + d), b = *reinterpret_cast<const v4f *>(row + d + 4);
            f = v8f{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        }
    }
    return f;
}

// ---------------------------------------------------------------- non-finite operands
//
// Weights of pairs that are not seen are 0, and 0 times an infinity or a NaN is NaN in a
// matrix product.  So where a workgroup has masked pairs in a tile, its waves first look
// through the tile that meets those weights (non_finite), and in the rare case take what is
// not finite out of it (Tile::clean) and put it back for the pairs that are seen: the forward
// kernel by what an infinity or a NaN does to a sum (add_non_finite), the backward kernels,
// whose tile enters the weights as well, a row at a time behind their loop (add_rows).

// Row bits of the tile's rows with an infinity or a NaN, the same in all waves of the
// workgroup.  words: LDS, [NW][ROWS / 32]; one barrier.
template <typename L, int ROWS, int NW>
__device__ __forceinline__ void non_finite(const uint8_t *t, uint32_t *words, uint32_t *bad)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int N = ROWS * L::kChunks / (64 * NW);
    uint32_t mine[ROWS / 32] = {};
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int slot = (wave * N + i) * 64 + lane, r = slot / L::kChunks;
        const uint32_t b = L::chunk_non_finite(*reinterpret_cast<const u4v *>(t + slot * 16)) ? 1u << (r & 31) : 0u;
#pragma unroll
        for (int x = 0; x < ROWS / 32; ++x) mine[x] |= (r >> 5) == x ? b : 0u;
    }
#pragma unroll
    for (int x = 0; x < ROWS / 32; ++x) {
        if (__any(mine[x] != 0)) {
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) mine[x] |= __shfl_xor(mine[x], d);
        }
        if (lane == 0) words[wave * (ROWS / 32) + x] = mine[x];
    }
    wait_lgkm();
    block_barrier();
#pragma unroll
    for (int x = 0; x < ROWS / 32; ++x) {
        bad[x] = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) bad[x] |= words[w * (ROWS / 32) + x];
        bad[x] = __builtin_amdgcn_readfirstlane(bad[x]);
    }
}

// word t of `bad` where t is the same in all lanes but not a constant
template <int N>
__device__ __forceinline__ uint32_t pick(const uint32_t *bad, int t)
{
    uint32_t w = bad[0];
#pragma unroll
    for (int x = 1; x < N; ++x) w = t == x ? bad[x] : w;
    return w;
}

// acc (rows d, column n) += the infinities and NaN of X's 32 rows from r0 that column n sees
// (bits of `seen`), times weights above zero: a count of them by matrix products
template <typename T, int DC, int DT>
__device__ __forceinline__ void add_non_finite(v16f *acc, uint32_t seen, uint32_t column_base, int r0, int h)
{
    const uint32_t bits = seen >> (4 * h);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        Frag<T> ones;
#pragma unroll
        for (int j = 0; j < 8; ++j) ones[j] = ((bits >> tile_row(8 * s + j, 0)) & 1) ? 1.f : 0.f;
#pragma unroll
        for (int dt = 0; dt < DC / 32; ++dt) {
            __builtin_amdgcn_sched_barrier(0);           // one tile at a time: registers, not speed
            const Frag<T> x = Tile<T, DT>::column_frag(column_base, r0 + 16 * s, dt);
            Frag<T> up, down;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = (float)x[j];
                const bool fin = fabsf(v) < INFINITY;
                up[j] = !fin && !(v == -INFINITY) ? 1.f : 0.f;
                down[j] = !fin && !(v == INFINITY) ? 1.f : 0.f;
            }
            const v16f zero = {};
            const v16f a = mma(up, ones, zero), b = mma(down, ones, zero);
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[dt][i] += (a[i] > 0.f ? INFINITY : 0.f) + (b[i] > 0.f ? -INFINITY : 0.f);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
}

// ---------------------------------------------------------------- masks

// What the masks leave between query positions [p0, p1] and keys [j0, j1]: nothing, some
// or all pairs; same: all are of one document.
struct Seen { bool any, all, same; };

// Range of the document numbers of some positions, and whether there is padding among them
// (negative numbers, which the range leaves out).  In memory: {lo, or ~lo with padding; hi}.
struct Documents {
    int lo, hi;
    bool padding;
};

__device__ __forceinline__ Seen classify(const AttentionMask &m, int prefix, int p0, int p1, int j0, int j1,
                                         const Documents &q, const Documents &k)
{
    bool any = true, all = true, same = true;
    if (m.causal) {
        any = j0 <= p1;
        all = j1 <= p0;
    }
    if (m.window) {
        any = any && p0 - j1 < m.window;
        all = all && p1 - j0 < m.window;
        if (!m.causal) {
            any = any && j0 - p1 < m.window;
            all = all && j1 - p0 < m.window;
        }
    }
    any = any || j0 < prefix;
    all = all || j1 < prefix;
    if (m.documents) {
        any = any && q.lo <= k.hi && k.lo <= q.hi;
        same = q.lo == q.hi && k.lo == k.hi && q.lo == k.lo && !q.padding && !k.padding;
        all = all && same;
    }
    return {any, all && any, same};
}

// A visited tile (-1: none): whether some pair of the workgroup is masked, whether this wave
// sees some and all pairs, and whether its pairs are of one document
struct Visit {
    int tile;
    bool part, any, all, same;
};

// Tiles of one loop axis that a workgroup visits, 64 at a time: lane t classifies tile
// base + t, and ballots hold what the workgroup and this wave see of them.
struct Schedule {
    uint64_t visit = 0, whole = 0, any = 0, all = 0, same = 0;
    int base = -64;
    // of the tile that next() gave: whether some pair of the workgroup is masked, whether this
    // wave sees some and all pairs
    bool part = false, wave_any = false, wave_all = false, wave_same = false;

    // next visited tile below `end`, or -1 (the same in all waves); f(tile) -> {of the
    // workgroup, of this wave}
    template <typename F>
    __device__ __forceinline__ int next(int end, F &&f)
    {
        while (!visit) {
            base += 64;
            if (base >= end) return -1;
            const int t = base + (threadIdx.x & 63);
            Seen g = {}, w = {};
            if (t < end) f(t, g, w);
            visit = __ballot(g.any);
            whole = __ballot(g.all);
            any = __ballot(w.any);
            all = __ballot(w.all);
            same = __ballot(w.same);
        }
        const int b = __builtin_ctzll(visit);
        visit &= visit - 1;
        part = !((whole >> b) & 1);
        wave_any = (any >> b) & 1;
        wave_all = (all >> b) & 1;
        wave_same = (same >> b) & 1;
        return base + b;
    }
    template <typename F>
    __device__ __forceinline__ Visit take(int end, F &&f)
    {
        const int t = next(end, f);
        return {t, part, wave_any, wave_all, wave_same};
    }
};

// LDS stages of a tile loop for tiles of so many bytes (both operands): three where they leave
// room for three workgroups a compute unit (loads then have two tiles' time: tiles of 64 keys and
// 64 dims in bfloat16 or 32 keys in float32), two, or one (float32, NARROW, more than 64 dims:
// the tiles of 128 rows fill the LDS)
constexpr int stages_of(int bytes) { return 3 * bytes <= 49152 ? 3 : 2 * bytes <= 131072 ? 2 : 1; }

// Keeps the order of the instructions before and after it
template <bool ON = true>
__device__ __forceinline__ void pin()
{
    if constexpr (ON) __builtin_amdgcn_sched_barrier(0);
}

// The loop over a workgroup's tiles: body(visit, stage) on each visited one, with fetch(stage,
// tile) two tiles ahead where there are three stages, one ahead with two, and after use with
// one; check(visit, stage) where some pair is masked.  LOADS: a thread's loads of a tile, at
// least.  Ends with no load under way, but without a barrier.
template <int NS, int LOADS, typename See, typename Fetch, typename Check, typename Body>
__device__ __forceinline__ void tile_loop(int end, See &&see, Fetch &&fetch, Check &&check, Body &&body)
{
    Schedule sched;
    Visit cur = sched.take(end, see), next = {};
    int stage = 0;
    if (cur.tile >= 0) {
        fetch(0, cur.tile);
        if constexpr (NS == 3) {
            next = sched.take(end, see);
            if (next.tile >= 0) fetch(1, next.tile);
        }
    }
    while (cur.tile >= 0) {
        if (NS == 3 && next.tile >= 0) wait_vmcnt<LOADS>();
        else wait_vmcnt<0>();
        block_barrier();
        const Visit ahead = NS == 3 && next.tile < 0 ? next : sched.take(end, see);
        if (NS > 1 && ahead.tile >= 0) fetch(NS == 3 ? (stage == 0 ? 2 : stage - 1) : stage ^ 1, ahead.tile);
        if (cur.part) check(cur, stage);
        if (cur.any) body(cur, stage);
        wait_lgkm();
        if constexpr (NS == 3) {
            cur = next;
            next = ahead;
            stage = stage == 2 ? 0 : stage + 1;
        } else {
            if (NS == 1 && ahead.tile >= 0) {
                block_barrier();
                fetch(0, ahead.tile);
            }
            cur = ahead;
            stage = NS == 1 ? 0 : stage ^ 1;
        }
    }
}

// Sum over the four waves of a workgroup of accumulators x (N tiles), left in wave 0; buf: LDS
// of 2 x N x 4096 bytes, which no wave still reads
template <int N>
__device__ __forceinline__ void join_waves(v16f *x, uint8_t *buf)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    v4f *at = reinterpret_cast<v4f *>(buf) + lane;
    auto put = [&](int k) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                at[((k * N + n) * 4 + g) * 64] = v4f{x[n][4 * g], x[n][4 * g + 1], x[n][4 * g + 2], x[n][4 * g + 3]};
    };
    auto add = [&](int k) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const v4f v = at[((k * N + n) * 4 + g) * 64];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[n][4 * g + i] += v[i];
            }
    };
    if (wave >= 2) put(wave - 2);
    __syncthreads();
    if (wave < 2) add(wave);
    __syncthreads();
    if (wave == 1) put(0);
    __syncthreads();
    if (wave == 0) add(0);
}

// Which of 32 neighbouring positions of the other side one position sees: bit r for position
// base + r.  Positions in [lo, hi) are seen, and on the queries' side those below the prefix.
struct Sight {
    int lo, hi, prefix, doc;

    static __device__ __forceinline__ uint32_t below(int n)
    {
        n = min(max(n, 0), 32);
        return n == 32 ? ~0u : (1u << n) - 1;
    }
    // docs: LDS, the document numbers of the 32 positions (null: no documents)
    __device__ __forceinline__ uint32_t word(int base, const int32_t *docs) const
    {
        uint32_t w = (below(hi - base) & ~below(lo - base)) | below(prefix - base);
        if (docs) {
            uint32_t same = 0;
#pragma unroll
            for (int r = 0; r < 32; r += 4) {
                const v4i d = *reinterpret_cast<const v4i *>(docs + r);
#pragma unroll
                for (int x = 0; x < 4; ++x) same |= d[x] == doc ? 1u << (r + x) : 0u;
            }
            w = doc >= 0 ? w & same : 0u;
        }
        return w;
    }
    // whether it sees position x, of document d
    __device__ __forceinline__ bool sees(int x, bool docs, int d) const
    {
        return ((x >= lo && x < hi) || x < prefix) && (!docs || (doc >= 0 && d == doc));
    }
};

// what query position p sees of len_k keys
__device__ __forceinline__ Sight query_sight(const AttentionMask &m, int p, int len_k, int prefix, int doc)
{
    Sight s;
    s.lo = m.window ? p - m.window + 1 : INT32_MIN / 2;
    s.hi = min(m.causal ? p + 1 : (m.window ? p + m.window : len_k), len_k);
    s.prefix = prefix;
    s.doc = doc;
    return s;
}
// the query positions that see key j
__device__ __forceinline__ Sight key_sight(const AttentionMask &m, int j, int len_k, int prefix, int doc)
{
    Sight s;
    s.lo = m.causal ? j : (m.window ? j - m.window + 1 : INT32_MIN / 2);
    s.hi = min(m.window ? j + m.window : len_k, len_k);
    if (j < prefix) {
        s.lo = INT32_MIN / 2;
        s.hi = len_k;
    }
    s.prefix = INT32_MIN / 2;
    s.doc = doc;
    return s;
}

// Whether bit tile_row(r, h) of a word is set, the word shifted right by 4 h beforehand
__device__ __forceinline__ bool word_bit(uint32_t w, int r) { return (w >> tile_row(r, 0)) & 1; }

// Documents of the positions [p0, p1] from the ranges of 64 positions; positions below zero
// have none
__device__ __forceinline__ Documents range_of(const int2 *ranges, int p0, int p1)
{
    Documents r = {INT32_MAX, -1, p0 < 0};
    for (int i = max(p0, 0) >> 6; i <= p1 >> 6; ++i) {
        const int2 s = ranges[i];
        r.lo = min(r.lo, s.x < 0 ? ~s.x : s.x);
        r.hi = max(r.hi, s.y);
        r.padding = r.padding || s.x < 0;
    }
    return r;
}

// Scores are kept as z, in units whose exponent of two is c z: z = s / (scale) and c =
// scale log2 e, or with a cap z = tanh and c = cap log2 e; a distance bias enters z as
// slope log2 e / c.
struct ScoreMap {
    float c, k1, slope;
};
__device__ __forceinline__ ScoreMap score_map(const AttentionMask &m, int hq)
{
    ScoreMap s;
    s.c = (m.cap > 0.f ? m.cap : m.scale) * kLog2e;
    s.k1 = m.cap > 0.f ? m.scale / m.cap : 1.f;
    s.slope = m.slopes ? m.slopes[hq] * kLog2e / s.c : 0.f;
    return s;
}

template <bool F32, int MODS>
__device__ __forceinline__ float tanh_of(float x)
{
    if constexpr (F32) return tanhf(x);
    // off by 2^-23 of 1
    const float t = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * (2.f * kLog2e)));
    if constexpr (MODS != kAnyCap) return t;
    // off by 2^-22 of itself: below 0.55 an odd polynomial (least relative error on that interval,
    // 2^-24.7, fitted to tanh(x) / x at Chebyshev points); above it the form above, which is there
    // more than half of 1
    const float y = x * x;
    const float p = fmaf(fmaf(fmaf(0.016458744f, y, -0.052684136f), y, 0.13320942f), y, -0.33332959f);
    return fabsf(x) < 0.55f ? fmaf(x, y * p, x) : t;
}

// 4 neighbouring elements to memory, rounded to nearest even for bf16
__device__ __forceinline__ void store4(float *p, float x0, float x1, float x2, float x3)
{
    *reinterpret_cast<v4f *>(p) = v4f{x0, x1, x2, x3};
}
__device__ __forceinline__ void store4(__bf16 *p, float x0, float x1, float x2, float x3)
{
    *reinterpret_cast<bf16x4 *>(p) = __builtin_convertvector(v4f{x0, x1, x2, x3}, bf16x4);
}

// a column of output tiles [d][column] times f into a row of memory
template <typename T, int DS>
__device__ __forceinline__ void store_columns(T *out, const v16f *x, float f, int h, int D)
{
#pragma unroll
    for (int dt = 0; dt < DS; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * dt + 8 * g + 4 * h;
            if (d < D) store4(out + d, x[dt][4 * g] * f, x[dt][4 * g + 1] * f, x[dt][4 * g + 2] * f, x[dt][4 * g + 3] * f);
        }
}

// Workgroup -> (head of batch, tile): each XCD takes a contiguous range of the heads, so
// that the keys and values of a head are read into one L2
__device__ __forceinline__ void head_tile(uint32_t bid, uint32_t n, uint32_t tiles, uint32_t &head, uint32_t &tile)
{
    const uint32_t xcd = bid % kXcds, local = bid / kXcds, per = n / kXcds, rem = n % kXcds;
    const uint32_t t = xcd * per + (xcd < rem ? xcd : rem) + local;
    head = t / tiles;
    tile = t % tiles;
}

}  // namespace
}  // namespace q2d
