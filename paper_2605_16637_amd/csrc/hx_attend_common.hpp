// What the kernels that look at cached keys share: number types, a sequence and its queries, which positions a query sees.
#pragma once

#include "hx_attend_args.hpp"

#include <type_traits>

namespace {

using AttendArgs = HxAttend;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

template <typename E> struct Types;
template <> struct Types<__bf16> { using x8 = bf16x8; using x4 = bf16x4; using x2 = bf16x2; };
template <> struct Types<_Float16> { using x8 = f16x8; using x4 = f16x4; using x2 = f16x2; };

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// 4 stored numbers of 8 bits; every e4m3 is a bf16 and an fp16 exactly
__device__ __forceinline__ void widen(uint32_t w, bf16x2 &a, bf16x2 &b)
{
    a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
}
__device__ __forceinline__ void widen(uint32_t w, f16x2 &a, f16x2 &b)
{
    a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
}

// 2 stored numbers of 4 bits, byte BYTE of w, times a power of 2 from a scale's byte; all of it is a bf16 and an fp16 exactly
template <int BYTE> __device__ __forceinline__ void widen4(uint32_t w, float unit, bf16x2 &a) { a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, BYTE); }
template <int BYTE> __device__ __forceinline__ void widen4(uint32_t w, float unit, f16x2 &a) { a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, unit, BYTE); }
// the 8 numbers of a word
template <typename X2> __device__ __forceinline__ void widen4(uint32_t w, float unit, X2 *x)
{
    widen4<0>(w, unit, x[0]); widen4<1>(w, unit, x[1]); widen4<2>(w, unit, x[2]); widen4<3>(w, unit, x[3]);
}
// 255 is NaN
__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte == 255 ? 0x7fc00000u : byte << 23); }

constexpr float NEG_INF = -__builtin_inff();
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float MAX_SLACK = 8.0f;            // a running maximum is raised when a score exceeds it by this many powers of 2
// Weights are taken this many powers of 2 up, in the products and the sums alike: the largest lie between 2^LIFT and 2^(LIFT + MAX_SLACK).
// fp16 ends at 2^-24 (a normal number at 2^-14): without it 32768 weights of 2^-25 of the largest were lost, 2^-10 together.  bf16 has fp32's range.
template <typename E> constexpr float LIFT = std::is_same_v<E, _Float16> ? 7.0f : 0.0f;

// Whether a sum of weights holds any: 0 where nothing was visible.  (A NaN among the visible has to reach the outputs.)
__device__ __forceinline__ bool holds_any(float l) { return l != 0.0f; }

// Whether a lane's sums hold an infinity or a NaN.
template <int N, typename F>
__device__ __forceinline__ bool any_odd(const F *o)
{
    uint32_t worst = 0;
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
        for (int i = 0; i < (int)(sizeof(F) / sizeof(float)); ++i) {
            const uint32_t size = __float_as_uint(o[x][i]) & 0x7fffffffu;
            worst = size > worst ? size : worst;
        }
    return worst >= 0x7f800000u;
}

// Bytes of a row of D numbers, without its scales.
template <int BITS, int D> constexpr int ROW = D * BITS / 8;

// How the keys of 16 rows go from memory into a matrix product: a lane's load, how many, and the place of the 8 numbers of the s-th of D / 32 operands.
template <int BITS, int D>
struct KeyPieces {
    static constexpr int BYTES = ROW<BITS, D> < 64 ? ROW<BITS, D> / 4 : 16, LOADS = ROW<BITS, D> / 4 / BYTES;
    static constexpr int NUMBERS = BYTES * 8 / BITS, EACH = NUMBERS / 8;         // of a load: numbers, operands
    using Piece = std::conditional_t<BYTES == 8, uint2, uint4>;
    static __device__ __forceinline__ int place(int s, int quad) { return (s / EACH) * (4 * NUMBERS) + quad * NUMBERS + (s % EACH) * 8; }
    // operand j of a load; exp: its scale's byte, of 4 bits
    template <typename E>
    static __device__ __forceinline__ typename Types<E>::x8 operand(const Piece &piece, uint32_t exp, int j)
    {
        using X8 = typename Types<E>::x8;
        if constexpr (BITS == 16) return __builtin_bit_cast(X8, piece);
        else {
            union { typename Types<E>::x2 x2[4]; X8 x8; } k;
            struct Words { uint32_t w[BYTES / 4]; } w = __builtin_bit_cast(Words, piece);
            if constexpr (BITS == 4) widen4(w.w[j], power_of(exp), k.x2);
            else { widen(w.w[2 * j], k.x2[0], k.x2[1]); widen(w.w[2 * j + 1], k.x2[2], k.x2[3]); }
            return k.x8;
        }
    }
};

// N stored numbers (N 4 or 8, of one group); exp: their scale's byte, of 4 bits only
template <typename E, int BITS, int N>
__device__ __forceinline__ void numbers(const char *from, const uint8_t *exp, float *to)
{
    using X2 = typename Types<E>::x2;
    if constexpr (BITS == 4) {
        X2 x[4];
        const uint32_t w = N == 8 ? *(const uint32_t *)from : *(const uint16_t *)from;
        widen4(w, power_of(*exp), x);
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = (float)x[i / 2][i % 2];
    } else if constexpr (BITS == 8) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            X2 a, b;
            widen(((const uint32_t *)from)[i], a, b);
            to[4 * i] = (float)a[0]; to[4 * i + 1] = (float)a[1]; to[4 * i + 2] = (float)b[0]; to[4 * i + 3] = (float)b[1];
        }
    } else
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = (float)((const E *)from)[i];
}

__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p; }

// 16 bytes a lane straight to LDS, a wavefront's beside each other from `to` on (the same for all lanes).  The compiler knows neither that the
// load is under way nor when it has come: that is waited for by count.
__device__ __forceinline__ void to_lds(uint32_t to, int off, const char *from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(from) : "memory");
}
__device__ __forceinline__ void to_lds(uint32_t to, const char *from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}

// the same of 4 bytes a lane
__device__ __forceinline__ void to_lds_word(uint32_t to, int off, const char *from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(off), "s"(from) : "memory");
}

constexpr int AT_THREADS = 256;
constexpr int MAX_SPLITS = 64;

// one value of the other half of the wavefront
__device__ __forceinline__ float other_half(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}

// value of the lane 16 away
__device__ __forceinline__ float lane_16_away(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(threadIdx.x & 16 ? r[0] : r[1]);
}

// A sequence and its queries.
struct Seq {
    int q0, nq, len, base;       // base: the position of the first query's token
    bool there, ok;              // queries lie within the call's; the rest is in range too
    const int32_t *table;
};

// pair: of sequence and KV head.  Where pages have been chosen for each query and KV head a "sequence" is one query, over a table of its own.
__device__ __forceinline__ Seq sequence(const AttendArgs &a, int pair)
{
    const KvView &kv = a.kv;
    const int i = pair / kv.n_heads;
    Seq s;
    if (a.picked) {
        const int len = a.picked_len[pair];                      // -1: the query is no sequence's
        s.q0 = i;
        s.nq = len < 0 ? 0 : 1;
        s.there = s.ok = true;
        s.len = len < 0 ? 0 : len;
        s.base = s.len - s.nq;
        s.table = a.picked + (int64_t)pair * a.picked_pages;
        return s;
    }
    s.q0 = a.q_ptr[i];
    const int q1 = a.q_ptr[i + 1], r = a.row ? a.row[i] : i;
    s.nq = q1 - s.q0;
    s.there = s.q0 >= 0 && q1 >= s.q0 && q1 <= a.n_q;
    s.ok = s.there && r >= 0 && r < kv.rows && s.nq <= a.max_q;
    s.len = s.ok ? kv.len[r] : 0;
    s.ok = s.ok && hx_row_ok(kv, r, s.len) && s.nq <= s.len;
    s.base = s.len - s.nq;
    s.table = hx_row(kv, s.ok ? r : 0);
    return s;
}

constexpr int ANC_WORDS = HX_MAX_DRAFTS / 32;
constexpr int TREE_BYTES = HX_MAX_DRAFTS * 4 * (1 + ANC_WORDS);

// Every draft's depth (-1: left out) and the bits of the drafts above it; s_parent: HX_MAX_DRAFTS words that are free yet.
__device__ __forceinline__ void plant(const AttendArgs &a, const Seq &q, int *s_parent, int *s_depth, uint32_t *s_anc)
{
    for (int i = threadIdx.x; i < q.nq; i += blockDim.x) s_parent[i] = a.parent[q.q0 + i];
    __syncthreads();
    for (int tid = threadIdx.x; tid < q.nq; tid += blockDim.x) {
        uint32_t mine[ANC_WORDS] = {};
        int depth = 0, at = tid;
        while (at >= 0) {
#pragma unroll
            for (int w = 0; w < ANC_WORDS; ++w) mine[w] |= at >> 5 == w ? 1u << (at & 31) : 0u;
            const int up = s_parent[at];
            if (up >= at || up < -2) { hx_raise(a.kv.status, HX_ERR_INDEX); at = -2; break; }
            at = up;
            ++depth;
        }
        s_depth[tid] = at == -2 ? -1 : depth - 1;
#pragma unroll
        for (int w = 0; w < ANC_WORDS; ++w) s_anc[tid * ANC_WORDS + w] = mine[w];
    }
    __syncthreads();
}

// The tiles of KEYS keys that some of the queries t_first .. t_last may see: the first sink_tiles, then those from lo_tile on.
struct Extent {
    int lo, hi, sink_tiles, lo_tile, n;
};

template <int KEYS>
__device__ __forceinline__ Extent extent(const AttendArgs &a, const Seq &q, int t_first, int t_last)
{
    const bool tree = a.parent != nullptr;
    Extent x{0, 0, 0, 0, 0};
    if (!q.ok || a.kv.n_pages == 0) return x;
    x.hi = tree ? q.len : q.base + t_last + 1;
    if (a.window > 0) {
        // the least position of a query: in a tree that of a draft without another above it, the first after the tokens before the drafts
        const int first_pos = tree ? q.base : q.base + t_first;
        x.lo = first_pos - a.window + 1;
        x.lo = x.lo > 0 ? x.lo : 0;
    }
    x.lo_tile = x.lo / KEYS;
    if (x.lo > 0) {
        const int sinks = a.n_sink < x.lo ? a.n_sink : x.lo;
        x.sink_tiles = (sinks + KEYS - 1) / KEYS;
        if (x.sink_tiles >= x.lo_tile) { x.sink_tiles = 0; x.lo_tile = 0; }
    }
    x.n = x.hi > 0 ? x.sink_tiles + (x.hi + KEYS - 1) / KEYS - x.lo_tile : 0;
    return x;
}

// Parts of n tiles: of `chunk` each, the last takes what is left.
__device__ __forceinline__ int parts_of(const AttendArgs &a, int n)
{
    const int parts = n > a.chunk ? (n + a.chunk - 1) / a.chunk : 1;
    return parts < a.splits ? parts : a.splits;
}

// A page that the pool has, or -1.
__device__ __forceinline__ int in_pool(const KvView &kv, int page)
{
    if (__builtin_amdgcn_ballot_w64(page >= kv.n_pages)) {
        if (page >= kv.n_pages) hx_raise(kv.status, HX_ERR_INDEX);
        page = page < kv.n_pages ? page : -1;
    }
    return page;
}

// What a lane's query sees.
struct Sight {
    bool tree, alive;
    int pos, t, base, nq, window, n_sink;
    const int *s_depth;
    const uint32_t *s_anc;
    __device__ __forceinline__ bool sees(int y) const
    {
        bool see = alive;
        int ypos = y;
        if (tree && y >= base) {
            const int d = y - base;
            const bool in = d < nq;
            see = see && in && ((s_anc[t * ANC_WORDS + ((in ? d : 0) >> 5)] >> (d & 31)) & 1);
            ypos = base + s_depth[in ? d : 0];
        }
        return see && ypos <= pos && (window <= 0 || ypos < n_sink || pos - ypos < window);
    }
};

__device__ __forceinline__ Sight sight(const AttendArgs &a, const Seq &q, int t, const int *s_depth, const uint32_t *s_anc)
{
    Sight v;
    v.tree = a.parent != nullptr;
    v.alive = q.ok && t < q.nq;
    v.t = v.alive ? t : 0;
    v.pos = q.base + t;
    if (v.tree && v.alive) {
        const int d = s_depth[t];
        v.alive = d >= 0;
        v.pos = q.base + d;
    }
    v.base = q.base; v.nq = q.nq; v.window = a.window; v.n_sink = a.n_sink; v.s_depth = s_depth; v.s_anc = s_anc;
    return v;
}

template <typename E>
__device__ __forceinline__ void put(E *to, bool wide, float a, float b, float c, float d)
{
    typename Types<E>::x4 y;
    y[0] = (E)a; y[1] = (E)b; y[2] = (E)c; y[3] = (E)d;
    if (wide) *(typename Types<E>::x4 *)to = y;
    else
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = y[j];
}

}  // namespace
