// Attention of a few or many queries over cached pages: sliding windows with sinks, trees of drafted tokens.
//
// One pass over the keys with a running maximum and sum.  The products are taken transposed, S^T = K Q^T and O^T = V^T P^T: a
// lane then holds one query's scores, its maximum needs one exchange between the two halves of the wavefront, the running
// maximum scales a lane's own accumulators, and the weights leave the first product in the very registers that the second wants them
// in (the order in which keys are summed is free, so the second product takes them in the first's order and the
// values are read from LDS in that order, transposed on the way).
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

// N stored numbers
template <typename E, bool FP8, int N>
__device__ __forceinline__ void numbers(const char *from, float *to)
{
    if constexpr (FP8) {
        using X2 = typename Types<E>::x2;
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

constexpr int AT_THREADS = 256;
constexpr int MAX_SPLITS = 64;

// one value of the other half of the wavefront
__device__ __forceinline__ float other_half(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}

// A sequence and its queries.
struct Seq {
    int q0, nq, len, base;       // base: the position of the first query's token
    bool there, ok;              // queries lie within the call's; the rest is in range too
    const int32_t *table;
};

__device__ __forceinline__ Seq sequence(const AttendArgs &a, int i)
{
    const KvView &kv = a.kv;
    Seq s;
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

// What workgroups leave for each other goes past the caches that they do not share: device-scope stores and loads, of 8 bytes.
__device__ __forceinline__ void leave(float *to, float x, float y)
{
    const uint64_t v = (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x);
    __hip_atomic_store((uint64_t *)to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 find(const float *from)
{
    const uint64_t v = __hip_atomic_load((const uint64_t *)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// The parts of a row tile put together by the workgroup that wrote the last of them.  Each workgroup writes its part, waits until
// it is written, and counts; who counts last reads all.  s: (2 parts + 1) ROWS floats; the others return.
template <typename E, int D, int ROWS>
__device__ __forceinline__ void join(const AttendArgs &a, const Seq &q, int pair, int rt, int parts, float *s)
{
    __shared__ int s_last;
    const int tid = threadIdx.x;
    const int64_t tile = (int64_t)pair * a.row_tiles + rt;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
        const int before = atomicAdd(a.done + tile, 1);
        s_last = before == parts - 1;
        if (s_last) __hip_atomic_store(a.done + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;
    const int head = pair % a.kv.n_heads;
    const int64_t slot0 = tile * a.splits * ROWS;
    const int rows_left = q.nq * a.group - rt * ROWS, rows = rows_left < ROWS ? rows_left : ROWS;
    const float v_unit = a.v_scale ? a.v_scale[a.layer * a.kv.n_heads + head] : 1.0f;
    // all parts' maxima and sums at once, then the factor of each part for each row
    float *s_l = s + (parts + 1) * ROWS;
    for (int u = tid; u < parts * rows; u += AT_THREADS) {
        const int p = u / rows, r = u % rows;
        const float2 ml = find((const float *)(a.part_ml + slot0 + (int64_t)p * ROWS + r));
        s[p * ROWS + r] = ml.x;
        s_l[p * ROWS + r] = ml.y;
    }
    __syncthreads();
    for (int r = tid; r < rows; r += AT_THREADS) {
        float top = NEG_INF, l = 0.0f;
        for (int p = 0; p < parts; ++p) top = fmaxf(top, s[p * ROWS + r]);
        const float use = top == NEG_INF ? 0.0f : top;
        for (int p = 0; p < parts; ++p) {
            const float y = s_l[p * ROWS + r], f = holds_any(y) ? __builtin_amdgcn_exp2f(s[p * ROWS + r] - use) : 0.0f;
            s[p * ROWS + r] = f;
            l += y * f;
        }
        s[parts * ROWS + r] = holds_any(l) ? v_unit / l : 0.0f;
        if (a.lse) {
            const int row = rt * ROWS + r;
            a.lse[(int64_t)(q.q0 + row / a.group) * a.n_heads + head * a.group + row % a.group] = holds_any(l) ? (top + __builtin_amdgcn_logf(l)) * LN2 : NEG_INF;
        }
    }
    __syncthreads();
    // four numbers of EACH rows a thread, AHEAD parts of each under way: a trip to the others' parts takes longer than all else here
    constexpr int EACH = 4, AHEAD = 4;
    const int all = rows * (D / 4);
    for (int u0 = tid; u0 < all; u0 += AT_THREADS * EACH) {
        float4 o[EACH];
        const float *from[EACH];
        int row[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int u = u0 + i * AT_THREADS < all ? u0 + i * AT_THREADS : u0;
            row[i] = u / (D / 4);
            from[i] = a.part + (slot0 + row[i]) * D + u % (D / 4) * 4;
            o[i] = make_float4(0, 0, 0, 0);
        }
        for (int p0 = 0; p0 < parts; p0 += AHEAD) {
            float2 x[EACH][AHEAD], y[EACH][AHEAD];
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (u0 + i * AT_THREADS < all)
#pragma unroll
                    for (int k = 0; k < AHEAD; ++k) {
                        const int p = p0 + k < parts ? p0 + k : parts - 1;
                        x[i][k] = find(from[i] + (int64_t)p * ROWS * D);
                        y[i][k] = find(from[i] + (int64_t)p * ROWS * D + 2);
                    }
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (u0 + i * AT_THREADS < all)
#pragma unroll
                    for (int k = 0; k < AHEAD; ++k) {
                        const float f = p0 + k < parts ? s[(p0 + k) * ROWS + row[i]] : 0.0f;
                        if (holds_any(f)) { o[i].x += x[i][k].x * f; o[i].y += x[i][k].y * f; o[i].z += y[i][k].x * f; o[i].w += y[i][k].y * f; }
                    }
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (u0 + i * AT_THREADS < all) {
                const int u = u0 + i * AT_THREADS, at = rt * ROWS + row[i];
                const float f = s[parts * ROWS + row[i]];
                put((E *)a.out + (int64_t)(q.q0 + at / a.group) * a.out_token + (int64_t)(head * a.group + at % a.group) * a.out_head + u % (D / 4) * 4, a.out_wide,
                    o[i].x * f, o[i].y * f, o[i].z * f, o[i].w * f);
            }
    }
}

// ---- many rows ---------------------------------------------------------------

constexpr int KT = 32;                                   // keys of a tile
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

constexpr int SPAN = 256;                                // tiles whose pages are looked up at once

// WR wavefronts beside each other take 32 rows each (a row: one query and query head of the KV head).
template <bool FP8, int D, int WR, bool PAGE16>
struct Tile {
    static constexpr int THREADS = 64 * WR;
    static constexpr int ROWS = 32 * WR;
    static constexpr int CH = D / 8;                     // 16-byte pieces of a row in LDS
    static constexpr int ROW_BYTES = FP8 ? D : 2 * D, PER_ROW = ROW_BYTES / 16;
    static constexpr int PIECES = KT * PER_ROW;          // of a tile's keys, or values
    static constexpr int LOADS = (PIECES + THREADS - 1) / THREADS;
    static constexpr int BUF = 2 * KT * D * 2;           // keys and values of a tile
    // Tiles in LDS.  What is stored in 16 bits goes there straight from memory; 8 bits pass through registers, where RING more are
    // under way.
    static constexpr bool DIRECT = !FP8 && PAGE16;
    static constexpr int RING = DIRECT && D < 256 ? 4 : 3;
    static constexpr int LDS = BUF * RING + SPAN * 16;
};

// Where 16-byte piece c of key row r lies in LDS.  Keys are read 32 rows at a time at one piece; the pieces of 8 rows and more fall in
// different banks.  Values are read as 4 rows x 64 bytes; those rows' pieces, too.  (The prompts' 8.5e6 LDS instructions count no bank conflict; 8 bits 6e4 of 1.3e7, as they are widened into LDS.)
template <int CH> __device__ __forceinline__ int k_piece(int r, int c) { return r * CH + (c ^ (r & (CH < 16 ? CH - 1 : 15))); }
template <int CH> __device__ __forceinline__ int v_piece(int r, int c) { return r * CH + (c ^ (CH >= 16 ? (r & 3) << 2 : ((r >> 1) & 1) << 2)); }

// PAGE16: pages of 16 tokens and more, so that what a wavefront loads at once lies in one page, and its address is a scalar.
//
// While a tile's weights are worked out the next tile's scores are: the matrix unit and the others are both busy within a wavefront, not
// only between two.
//
// A tile is 16 products of 32 cycles a wavefront, 16 KB that it reads from LDS at 128 bytes a cycle and CU, and some 130 other instructions, 16
// of them exponentials of 16 cycles: for the 8 wavefronts of a CU 1024 cycles of the matrix units, 1024 of LDS, some 1300 of the rest.
// They take 2800, so two wavefronts a SIMD fill half of each other's waits.  Prompts of 2310, 3010 and 2893 tokens, window 2048, 32 heads of 128:
// 216 us, 0.80 PFLOP/s (a bf16 product of 8192^3 here: 1.18; cards differ, up to 244).  24 trees of up to 25 drafts over some 2400 tokens: 76 us + 10 to join, and 16
// trees of up to 64 over 8 bits and some 16500 tokens 468 us, 0.42 PFLOP/s: 8 bits pass through registers and are widened on their way to LDS.  Measured and
// not taken: 64 rows a wavefront at one wavefront a SIMD, which halves what is read from LDS (495 and 882 us); operands read a stage ahead
// (221 and 490, where what is here took 220 and 473).
template <typename E, bool FP8, int D, int WR, bool PAGE16>
__global__ __launch_bounds__(64 * WR, D == 256 ? 1 : D == 64 && !FP8 && PAGE16 ? 3 : 2) void hx_attend_kernel(AttendArgs a)
{
    using X8 = typename Types<E>::x8;
    using X2 = typename Types<E>::x2;
    using C = Tile<FP8, D, WR, PAGE16>;
    constexpr int RING = C::RING, CH = C::CH, LOADS = C::LOADS, THREADS = C::THREADS, ROW_BYTES = C::ROW_BYTES, PER_ROW = C::PER_ROW;
    extern __shared__ __align__(16) char smem[];
    longlong2 *s_off = (longlong2 *)(smem + C::BUF * RING);
    int *s_depth = (int *)(smem + C::LDS);
    uint32_t *s_anc = (uint32_t *)(s_depth + HX_MAX_DRAFTS);     // [HX_MAX_DRAFTS][ANC_WORDS]

    const KvView &kv = a.kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, col = lane & 31;
    const int nh = a.n * kv.n_heads;
    const int pair = blockIdx.x % nh, rest = blockIdx.x / nh;
    // row tiles of the same keys beside each other: they meet in the XCD's cache
    const int split = rest / a.row_tiles, rt = a.row_tiles - 1 - rest % a.row_tiles;
    const int head = pair % kv.n_heads;
    const Seq sq = sequence(a, pair / kv.n_heads);
    if (!sq.there) { if (tid == 0) hx_raise(kv.status, HX_ERR_INDEX); return; }
    if (rt * C::ROWS >= sq.nq * (int64_t)a.group) return;
    if (!sq.ok && tid == 0) hx_raise(kv.status, HX_ERR_INDEX);
    const int base = sq.base;
    const bool tree = a.parent != nullptr;

    const int t_first = rt * C::ROWS / a.group;
    int t_last = (rt * C::ROWS + C::ROWS - 1) / a.group;
    t_last = t_last < sq.nq ? t_last : sq.nq - 1;
    const Extent ex = extent<KT>(a, sq, t_first, t_last);
    const int parts = parts_of(a, ex.n);
    if (split >= parts) return;
    const int tile0 = split * a.chunk, tile1 = split == parts - 1 ? ex.n : tile0 + a.chunk;
    if (tree && sq.ok) plant(a, sq, (int *)smem, s_depth, s_anc);

    // this lane's row
    const int row = rt * C::ROWS + wave * 32 + col, t = row / a.group, qhead = head * a.group + row % a.group;
    const Sight view = sight(a, sq, t, s_depth, s_anc);

    const float k_unit = a.k_scale ? a.k_scale[a.layer * kv.n_heads + head] : 1.0f;
    const float sc = a.scale * k_unit * LOG2E;
    // the score's sign goes into the query, and its factor is no 0: a masked score stays -infinity
    const float c = fmaxf(fabsf(sc), 1e-37f);
    X8 qf[D / 16];
    {
        const E *qp = (const E *)a.q + (int64_t)(sq.q0 + t) * a.q_token + (int64_t)qhead * a.q_head;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            X8 x = {};
            if (view.alive) {
                if (a.q_wide) x = *(const X8 *)(qp + s * 16 + half * 8);
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = qp[s * 16 + half * 8 + i];
            }
            if (sc < 0)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = -x[i];
            qf[s] = x;
        }
    }

    // Tiles that all rows of this wavefront see whole: their first key is at most whole_to, and at least whole_from or at most whole_sink.
    const int wave_first = tree ? base - 1 : base + (rt * C::ROWS + wave * 32) / a.group;
    const int wave_last = tree ? sq.len : base + (rt * C::ROWS + wave * 32 + 31) / a.group;
    const int whole_to = wave_first + 1 - KT, whole_from = a.window > 0 ? wave_last - a.window + 1 : 0, whole_sink = a.n_sink - KT;
    const bool rows_here = rt * C::ROWS + wave * 32 < sq.nq * a.group;           // else the wavefront only loads

    const int beyond_sinks = (ex.lo_tile - ex.sink_tiles) * KT;
    auto start_of = [&](int tile) { return tile * KT + (tile < ex.sink_tiles ? 0 : beyond_sinks); };
    auto page_at = [&](int y) {
        const int page = y < ex.hi ? sq.table[y >> kv.shift] : -1;
        if (page >= kv.n_pages) hx_raise(kv.status, HX_ERR_INDEX);
        return page < kv.n_pages ? page : -1;
    };
    auto in_sight = [&](int y) { return y < ex.hi && (y >= ex.lo || y < a.n_sink); };       // of some row of the tile of rows

    uint4 rk[C::DIRECT ? 1 : RING][LOADS], rv[C::DIRECT ? 1 : RING][LOADS];
    uint32_t there[RING], now = 0;                       // which keys of the tiles under way are there, and of the one whose scores are next
    const int64_t page_bytes = ((int64_t)kv.n_heads << kv.shift) * ROW_BYTES;
    const int64_t here = (int64_t)a.layer * kv.n_pages * page_bytes + ((int64_t)head << kv.shift) * ROW_BYTES;
    const char *k_at = (const char *)kv.k + here, *v_at = (const char *)kv.v + here;
    const int in_page = (1 << kv.shift) - 1;
    const int my_key = tid / PER_ROW, my_part = tid % PER_ROW;
    const bool loads = C::PIECES % THREADS == 0 || wave * 64 < C::PIECES;
    // A tile's keys and values are asked for, by the same number of loads whatever the tile, so that it is known how many are under way.
    // Through registers what is not there is read from the pool's start and cleared on its way to LDS.  Straight to LDS a lane's 16 bytes
    // lie in the order of the lanes: each asks for the piece that belongs there, zeros where nothing is.
    int k_off[LOADS], v_off[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        const int key = j * THREADS / PER_ROW + my_key, in_group = key - (j * THREADS / PER_ROW + wave * 64 / PER_ROW);
        k_off[j] = C::DIRECT ? in_group * ROW_BYTES + (k_piece<CH>(key, my_part) - key * CH) * 16 : lane * 16;
        v_off[j] = C::DIRECT ? in_group * ROW_BYTES + (v_piece<CH>(key, my_part) - key * CH) * 16 : lane * 16;
    }
    const uint32_t lds0 = lds_address(smem);
    // two: where the tile's first and second 16 keys lie, the lowest bit set where some key of the tile is not there, -1 where no page is
    auto ask = [&](int tile, longlong2 two, auto set) {
        constexpr int S = decltype(set)::value;
        const int64_t o0 = uniform(two.x), o1 = uniform(two.y);
        const int y0 = start_of(tile);
        const bool whole = PAGE16 && !((o0 | o1) & 1);
        auto place_of = [&](int key) -> int64_t {
            const int y = y0 + key;
            if (tile >= tile1 || key >= KT || !in_sight(y)) return -1;
            if constexpr (PAGE16) {
                const int64_t o = key < 16 ? o0 : o1;
                return o < 0 ? -1 : (o & ~(int64_t)15) + (key & 15) * ROW_BYTES;
            }
            const int page = page_at(y);
            return page < 0 ? -1 : page * page_bytes + (y & in_page) * ROW_BYTES;
        };
        there[S] = 0xffffffffu;
        if (!whole) there[S] = (uint32_t)__builtin_amdgcn_ballot_w64(place_of(col) >= 0);
        if constexpr (C::DIRECT) {
            if (loads)
#pragma unroll
                for (int j = 0; j < LOADS; ++j) {
                    const int key = j * THREADS / PER_ROW + my_key, first = (j * THREADS / PER_ROW + wave * 64 / PER_ROW) & 31;
                    const uint32_t to = lds0 + S * C::BUF + (j * THREADS + wave * 64) * 16, to_v = to + KT * CH * 16;
                    if (whole) {
                        const int64_t at = (first < 16 ? o0 : o1) + (first & 15) * ROW_BYTES;
                        to_lds(to, k_off[j], k_at + at);
                        to_lds(to_v, v_off[j], v_at + at);
                    } else {
                        const int64_t at = place_of(key);
                        to_lds(to, at >= 0 ? k_at + at + (k_piece<CH>(key, my_part) - key * CH) * 16 : (const char *)a.zeros);
                        to_lds(to_v, at >= 0 ? v_at + at + (v_piece<CH>(key, my_part) - key * CH) * 16 : (const char *)a.zeros);
                    }
                }
        } else {
            int64_t at[LOADS];
            if (whole)
#pragma unroll
                for (int j = 0; j < LOADS; ++j) {
                    const int first = (j * THREADS / PER_ROW + wave * 64 / PER_ROW) & 31;
                    at[j] = (first < 16 ? o0 : o1) + (first & 15) * ROW_BYTES + lane * 16;
                }
            else
#pragma unroll
                for (int j = 0; j < LOADS; ++j) {
                    const int64_t x = place_of(j * THREADS / PER_ROW + my_key);
                    at[j] = x >= 0 ? x + my_part * 16 : 0;
                }
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                rk[S][j] = *(const uint4 *)(k_at + at[j]);
                rv[S][j] = *(const uint4 *)(v_at + at[j]);
            }
        }
    };
    auto store = [&](auto set) {
        constexpr int S = decltype(set)::value;
        uint4 *sk = (uint4 *)(smem + S * C::BUF), *sv = sk + KT * CH;
        if (!loads) return;
        if (there[S] != 0xffffffffu)
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                if (!((there[S] >> (i * THREADS / PER_ROW + my_key)) & 1)) rk[S][i] = rv[S][i] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int key = i * THREADS / PER_ROW + my_key;
            if constexpr (FP8) {
                union { X2 x[8]; uint4 u[2]; } wk, wv;
                const uint32_t kk[4] = {rk[S][i].x, rk[S][i].y, rk[S][i].z, rk[S][i].w}, vv[4] = {rv[S][i].x, rv[S][i].y, rv[S][i].z, rv[S][i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) { widen(kk[j], wk.x[2 * j], wk.x[2 * j + 1]); widen(vv[j], wv.x[2 * j], wv.x[2 * j + 1]); }
                // half of a row's lanes begin with their second piece: 8 lanes beside each other fill all banks
                const bool second = my_part & 4;
                const int at0 = 2 * my_part + second, at1 = at0 ^ 1;
                auto either = [&](const uint4 &x, const uint4 &y) { return make_uint4(second ? y.x : x.x, second ? y.y : x.y, second ? y.z : x.z, second ? y.w : x.w); };
                const uint4 k0 = wk.u[0], k1 = wk.u[1], v0 = wv.u[0], v1 = wv.u[1];
                sk[k_piece<CH>(key, at0)] = either(k0, k1); sk[k_piece<CH>(key, at1)] = either(k1, k0);
                sv[v_piece<CH>(key, at0)] = either(v0, v1); sv[v_piece<CH>(key, at1)] = either(v1, v0);
            } else {
                sk[k_piece<CH>(key, my_part)] = rk[S][i];
                sv[v_piece<CH>(key, my_part)] = rv[S][i];
            }
        }
    };

    f32x16 o[D / 32] = {}, s = {};
    float m = NEG_INF, l = 0.0f, l1 = 0.0f;
    // This lane's places in a tile of the first ring place.  A key's pieces 2 x + half are one x apart in the bits that x has; its values: 4 keys
    // x 16 numbers a group of 16 lanes, of which lane j reads 4 numbers of key j / 4 and gets number j of the 4 keys.
    uint32_t k_lane[D / 16], v_lane[D / 32];
#pragma unroll
    for (int x = 0; x < D / 16; ++x) k_lane[x] = lds0 + k_piece<CH>(col, 2 * x + half) * 16;
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
        v_lane[x] = lds0 + KT * CH * 16 + v_piece<CH>(4 * half + ((lane & 15) >> 2), x * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) * 16 + (lane & 1) * 8;
    auto scores = [&](auto set) {
        constexpr int S = decltype(set)::value;
        f32x16 acc = {};
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
            using LdsPtr = __attribute__((address_space(3))) const X8 *;
            acc = mfma32(*(LdsPtr)(uintptr_t)(k_lane[x] + S * C::BUF), qf[x], acc);
        }
        return acc;
    };

    int seg0 = tile0, seg1 = tile0;                      // tiles whose places are in s_off
    auto place = [&](int tile) { return PAGE16 && tile < seg1 ? s_off[tile - seg0] : longlong2{-1, -1}; };
    auto one_tile = [&](int tile, auto set) {
        constexpr int S = decltype(set)::value, NEXT = (S + 1) % RING;
        using Next = std::integral_constant<int, NEXT>;
        const uint32_t seen = now;
        now = there[NEXT];
        const longlong2 two = place(C::DIRECT ? tile + RING - 1 : tile + 1 + RING);
        if constexpr (C::DIRECT) {
            // the next tile has come, those after it may be under way; the place of the one before this is free once all are here
            if (tile + RING - 2 < seg1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LOADS * (RING - 3)) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tile + RING - 1 < seg1) ask(tile + RING - 1, two, std::integral_constant<int, (S + RING - 1) % RING>{});
        } else {
            // the next tile's registers go to LDS and are free for the one RING further on
            store(Next{});
            ask(tile + 1 + RING, two, Next{});
            __syncthreads();
        }
        if (!rows_here || tile >= seg1) return;
        // a lane's register i is the score of key y0 + 8 (i / 4) + 4 half + i % 4
        const int y0 = start_of(tile);
        if (seen != 0xffffffffu || y0 > whole_to || (y0 < whole_from && y0 > whole_sink)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int k = 8 * (i / 4) + 4 * half + i % 4;
                s[i] = ((seen >> k) & 1) && view.sees(y0 + k) ? s[i] : NEG_INF;
            }
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(top, other_half(top)) * c;
        if (__builtin_amdgcn_ballot_w64(top > m + (MAX_SLACK + LIFT<E>))) {
            const float m_new = fmaxf(m, top - LIFT<E>);
            const float shrink = __builtin_amdgcn_exp2f(m - (m_new == NEG_INF ? 0.0f : m_new));
            m = m_new;
            l *= shrink;
            l1 *= shrink;
#pragma unroll
            for (int x = 0; x < D / 32; ++x) o[x] *= shrink;
        }
        const float m_use = m == NEG_INF ? 0.0f : m;
        // (after the last tile the scores of what happens to lie in LDS, which nobody asks for)
        const f32x16 next = scores(Next{});
        union { X8 x8[2]; X2 x2[8]; } p;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float w0 = __builtin_amdgcn_exp2f(fmaf(s[2 * i], c, -m_use)), w1 = __builtin_amdgcn_exp2f(fmaf(s[2 * i + 1], c, -m_use));
            p.x2[i][0] = (E)w0;
            p.x2[i][1] = (E)w1;
            l += w0;
            l1 += w1;
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                using LdsPtr = __attribute__((address_space(3))) i16x4 *;
                union { i16x4 h[2]; X8 x; } vf;
                vf.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(uintptr_t)(v_lane[x] + S * C::BUF + st * 16 * CH * 16));
                vf.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(uintptr_t)(v_lane[x] + S * C::BUF + (st * 16 + 8) * CH * 16));
                o[x] = mfma32(vf.x, p.x8[st], o[x]);
            }
        }
        s = next;
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I3 = std::integral_constant<int, RING == 4 ? 3 : 0>;
    for (seg0 = tile0; seg0 < tile1; seg0 = seg1) {
        // the places of the next SPAN tiles, which then need not be waited for among the keys
        seg1 = seg0 + SPAN < tile1 ? seg0 + SPAN : tile1;
        if constexpr (PAGE16) {
            if (seg0 > tile0) __syncthreads();
            for (int i = tid; i < 2 * (seg1 - seg0); i += THREADS) {
                const int y0 = start_of(seg0 + i / 2), y = y0 + (i & 1) * 16, page = page_at(y);
                const bool all = y0 + KT <= ex.hi && (y0 >= ex.lo || y0 + KT <= a.n_sink);
                ((int64_t *)s_off)[i] = page < 0 ? -1 : (page * page_bytes + (y & in_page) * ROW_BYTES) | (all ? 0 : 1);
            }
        }
        __syncthreads();
        ask(seg0, place(seg0), I0{});
        if (!C::DIRECT || seg0 + 1 < seg1) ask(seg0 + 1, place(seg0 + 1), I1{});
        if (!C::DIRECT || (RING == 4 && seg0 + 2 < seg1)) ask(seg0 + 2, place(seg0 + 2), I2{});
        now = there[0];
        if constexpr (C::DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        else {
            store(I0{});
            ask(seg0 + 3, place(seg0 + 3), I0{});
        }
        __syncthreads();
        s = scores(I0{});
        for (int tile = seg0; tile < seg1; tile += RING) {
            one_tile(tile, I0{});
            one_tile(tile + 1, I1{});
            one_tile(tile + 2, I2{});
            if constexpr (RING == 4) one_tile(tile + 3, I3{});
        }
    }

    l += l1;
    l += other_half(l);
    // A weight of 0 times an infinite or NaN value is no 0: where a row's sums are not finite they are taken again key by key, from what it
    // sees alone, with weights of 32 bits, which an infinite value leaves infinite.
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(any_odd<D / 32>(o)) != 0, false)) {
        const float m_use = m == NEG_INF ? 0.0f : m;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) o[x] = f32x16{};
#pragma unroll 1
        for (int key = tile0 * KT; key < tile1 * KT; ++key) {
            const int y = start_of(key / KT) + key % KT, page = in_sight(y) ? page_at(y) : -1;
            if (page < 0) continue;
            const int64_t at = page * page_bytes + (y & in_page) * ROW_BYTES;
            float dot = 0.0f;
#pragma unroll
            for (int x = 0; x < D / 16; ++x) {
                float k[8];
                numbers<E, FP8, 8>(k_at + at + (x * 16 + half * 8) * (ROW_BYTES / D), k);
#pragma unroll
                for (int i = 0; i < 8; ++i) dot = fmaf((float)qf[x][i], k[i], dot);
            }
            dot += other_half(dot);
            const bool see = view.sees(y);
            const float weight = __builtin_amdgcn_exp2f(fmaf(dot, c, -m_use));
#pragma unroll
            for (int x = 0; x < D / 32; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v[4];
                    numbers<E, FP8, 4>(v_at + at + (x * 32 + 8 * i + 4 * half) * (ROW_BYTES / D), v);
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[x][4 * i + j] += see ? weight * v[j] : 0.0f;
                }
        }
    }
    if (!view.alive) { m = NEG_INF; l = 0.0f; }
    if (t >= sq.nq) return;
    if (parts > 1) {
        const int64_t slot = (((int64_t)pair * a.row_tiles + rt) * a.splits + split) * C::ROWS + wave * 32 + col;
        float *to = a.part + slot * D;
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(float4 *)(to + x * 32 + 8 * i + 4 * half) = make_float4(o[x][4 * i], o[x][4 * i + 1], o[x][4 * i + 2], o[x][4 * i + 3]);
        if (half == 0) a.part_ml[slot] = make_float2(m, l);
        return;
    }
    const float v_unit = a.v_scale ? a.v_scale[a.layer * kv.n_heads + head] : 1.0f;
    const float f = holds_any(l) ? v_unit / l : 0.0f;
    E *to = (E *)a.out + (int64_t)(sq.q0 + t) * a.out_token + (int64_t)qhead * a.out_head;
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = holds_any(l) ? o[x][4 * i + j] * f : 0.0f;
            put(to + x * 32 + 8 * i + 4 * half, a.out_wide, y[0], y[1], y[2], y[3]);
        }
    if (a.lse && half == 0) a.lse[(int64_t)(sq.q0 + t) * a.n_heads + qhead] = holds_any(l) ? (m + __builtin_amdgcn_logf(l)) * LN2 : NEG_INF;
}

// The parts of rows put together, by D / 4 lanes a row: each has 4 of its numbers, and the maximum and sum of some of its parts.
template <typename E, int D, int KEYS, int ROWS>
__global__ __launch_bounds__(AT_THREADS) void hx_attend_join_kernel(AttendArgs a)
{
    constexpr int G = D / 4, TOGETHER = AT_THREADS / G, KEEP = (MAX_SPLITS + G - 1) / G;
    const int per_tile = ROWS / TOGETHER, pair = blockIdx.x / (a.row_tiles * per_tile), rt = blockIdx.x / per_tile % a.row_tiles;
    const int r = blockIdx.x % per_tile * TOGETHER + threadIdx.x / G, g = threadIdx.x % G, row = rt * ROWS + r;
    const Seq sq = sequence(a, pair / a.kv.n_heads);
    if (!sq.ok || rt * ROWS >= sq.nq * (int64_t)a.group) return;
    int t_last = (rt * ROWS + ROWS - 1) / a.group;
    t_last = t_last < sq.nq ? t_last : sq.nq - 1;
    const int parts = parts_of(a, extent<KEYS>(a, sq, rt * ROWS / a.group, t_last).n), t = row / a.group, head = pair % a.kv.n_heads;
    if (parts == 1 || t >= sq.nq) return;                        // (rows beside each other in a wavefront may end here)
    const int64_t slot0 = ((int64_t)pair * a.row_tiles + rt) * a.splits * ROWS + r;
    float2 ml[KEEP];
    float top = NEG_INF;
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
        const int p = k * G + g;
        ml[k] = p < parts ? a.part_ml[slot0 + (int64_t)p * ROWS] : make_float2(NEG_INF, 0.0f);
        top = fmaxf(top, ml[k].x);
    }
#pragma unroll
    for (int d = G / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, G));
    const float use = top == NEG_INF ? 0.0f : top;
    float f[KEEP], l = 0.0f;
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
        f[k] = holds_any(ml[k].y) ? __builtin_amdgcn_exp2f(ml[k].x - use) : 0.0f;
        l += ml[k].y * f[k];
    }
#pragma unroll
    for (int d = G / 2; d > 0; d >>= 1) l += __shfl_xor(l, d, G);
    float4 o = make_float4(0, 0, 0, 0);
    for (int p0 = 0; p0 < parts; p0 += 8) {
        float4 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = *(const float4 *)(a.part + (slot0 + (int64_t)(p0 + i < parts ? p0 + i : parts - 1) * ROWS) * D + 4 * g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int p = p0 + i;
            float w = __shfl(f[0], p % G, G);
#pragma unroll
            for (int k = 1; k < KEEP; ++k) {
                const float v = __shfl(f[k], p % G, G);
                w = p / G == k ? v : w;
            }
            if (p < parts && holds_any(w)) { o.x += x[i].x * w; o.y += x[i].y * w; o.z += x[i].z * w; o.w += x[i].w * w; }
        }
    }
    const float v_unit = a.v_scale ? a.v_scale[a.layer * a.kv.n_heads + head] : 1.0f, unit = holds_any(l) ? v_unit / l : 0.0f;
    const int qhead = head * a.group + row % a.group;
    put((E *)a.out + (int64_t)(sq.q0 + t) * a.out_token + (int64_t)qhead * a.out_head + 4 * g, a.out_wide, o.x * unit, o.y * unit, o.z * unit, o.w * unit);
    if (a.lse && g == 0) a.lse[(int64_t)(sq.q0 + t) * a.n_heads + qhead] = holds_any(l) ? (top + __builtin_amdgcn_logf(l)) * LN2 : NEG_INF;
}

// ---- few rows ----------------------------------------------------------------

// value of the lane 16 away
__device__ __forceinline__ float lane_16_away(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(threadIdx.x & 16 ? r[0] : r[1]);
}

template <int CH> __device__ __forceinline__ int few_v_piece(int r, int c) { return r * CH + (c ^ (CH >= 16 ? (r & 7) << 1 : ((r >> 1) & 3) << 1)); }

constexpr int FEW_KEYS = 32;

// LDS of a wavefront: a tile's values, and at the end its sums
constexpr int few_wave_lds(int dim, int cols) { return FEW_KEYS * dim * 2 > 16 * cols * dim * 4 ? FEW_KEYS * dim * 2 : 16 * cols * dim * 4; }

// Up to 16 COLS rows of a KV head, as single tokens bring them: bound by the reads of keys and values.  Each wavefront takes every fourth tile
// of 32 keys by itself, with nothing shared until the end: the keys go from memory into the registers of the matrix product, the values
// through its own piece of LDS, which transposes them; what it asks for next is under way all the time.  256 sequences, window 4096, one token each,
// 8 KV heads of 128: 600 us, 5.8 TB/s (a plain copy: 4.7).  One sequence is launch, lookups and three round trips: a token of 230 10 us, 8
// drafts over 856 18 us, of which the parts' joining some 4.
//
// A weight is two numbers of q's type, its rounding and what that leaves, in a product each: what remains of its rounding is 2^-16 of it (fp16
// 2^-22), so that the result is as near the exact one as its own rounding lets it be.  With one number a result of 16 bits was off by 1.3 to 1.4
// times as much.  What the second product costs: 0 to 2 % in most cases, up to 7 where an 8-bit cache or heads of 64 bring fewer bytes a weight
// and rows are more than 16.  (The kernel for many rows, which the matrix units and the weights' arithmetic bound, has one number: two
// took 9 to 29 % longer, 24 trees of 25 drafts 84 -> 94 us, the prompts above 213 -> 262.)
template <typename E, bool FP8, int D, int COLS, bool PAGE16>
__global__ __launch_bounds__(AT_THREADS, D == 256 ? 1 : COLS == 1 && D == 64 ? 4 : COLS == 1 && FP8 ? 3 : 2) void hx_attend_few_kernel(AttendArgs a)
{
    using X8 = typename Types<E>::x8;
    using X2 = typename Types<E>::x2;
    constexpr int CH = D / 8, ROW_BYTES = FP8 ? D : 2 * D;
    constexpr int K_LOADS = ROW_BYTES / 64;                     // of a lane for 16 keys
    constexpr int V_LOADS = FEW_KEYS * ROW_BYTES / 1024;        // of a lane for the tile
    constexpr int PER_ROW = ROW_BYTES / 16;
    constexpr int WAVE_LDS = few_wave_lds(D, COLS), ROWS = 16 * COLS;
    extern __shared__ __align__(16) char smem[];
    int *s_depth = (int *)(smem + 4 * WAVE_LDS);
    uint32_t *s_anc = (uint32_t *)(s_depth + HX_MAX_DRAFTS);
    __shared__ float s_ml[4][2][ROWS];

    const KvView &kv = a.kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), quad = lane >> 4, col = lane & 15;
    const int nh = a.n * kv.n_heads;
    const int pair = blockIdx.x % nh, split = blockIdx.x / nh, head = pair % kv.n_heads;
    const Seq sq = sequence(a, pair / kv.n_heads);
    if (!sq.there) { if (tid == 0) hx_raise(kv.status, HX_ERR_INDEX); return; }
    if (sq.nq == 0) return;
    if (!sq.ok && tid == 0) hx_raise(kv.status, HX_ERR_INDEX);
    const int base = sq.base;
    const bool tree = a.parent != nullptr;
    const Extent ex = extent<FEW_KEYS>(a, sq, 0, sq.nq - 1);
    const int parts = parts_of(a, ex.n);
    if (split >= parts) return;
    const int tile0 = split * a.chunk, tile1 = split == parts - 1 ? ex.n : tile0 + a.chunk;
    if (tree && sq.ok) plant(a, sq, (int *)smem, s_depth, s_anc);

    const float k_unit = a.k_scale ? a.k_scale[a.layer * kv.n_heads + head] : 1.0f;
    const float sc = a.scale * k_unit * LOG2E;
    const float c = fmaxf(fabsf(sc), 1e-37f);
    // this lane's rows, one of each block of 16
    int t[COLS], qhead[COLS];
    Sight view[COLS];
    X8 qf[COLS][D / 32];
#pragma unroll
    for (int w = 0; w < COLS; ++w) {
        t[w] = (16 * w + col) / a.group;
        qhead[w] = head * a.group + (16 * w + col) % a.group;
        view[w] = sight(a, sq, t[w], s_depth, s_anc);
        const E *qp = (const E *)a.q + (int64_t)(sq.q0 + t[w]) * a.q_token + (int64_t)qhead[w] * a.q_head;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            // which 8 numbers of a row a lane's s-th piece of a key holds
            const int d = FP8 ? (s >> 1) * 64 + quad * 16 + (s & 1) * 8 : s * 32 + quad * 8;
            X8 x = {};
            if (view[w].alive) {
                if (a.q_wide) x = *(const X8 *)(qp + d);
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = qp[d + i];
            }
            if (sc < 0)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = -x[i];
            qf[w][s] = x;
        }
    }
    int all_last = base + sq.nq - 1;
    if (tree) all_last = sq.len;

    auto start_of = [&](int tile) { return (tile < ex.sink_tiles ? tile : tile - ex.sink_tiles + ex.lo_tile) * FEW_KEYS; };
    auto page_of = [&](int tile) {
        const int y = start_of(tile) + (lane & 31);
        int page = -1;
        if (tile < tile1 && y < ex.hi && (y >= ex.lo || y < a.n_sink)) page = sq.table[y >> kv.shift];
        return page;
    };
    const int64_t page_bytes = ((int64_t)kv.n_heads << kv.shift) * ROW_BYTES;
    const int64_t here = (int64_t)a.layer * kv.n_pages * page_bytes + ((int64_t)head << kv.shift) * ROW_BYTES;
    const char *k_at = (const char *)kv.k + here, *v_at = (const char *)kv.v + here;
    const int in_page = (1 << kv.shift) - 1;
    uint4 rk[2][K_LOADS], rv[V_LOADS];
    auto fetch_k = [&](int tile, int pages, bool whole) {
        const int y0 = start_of(tile), off = col * ROW_BYTES + quad * 16;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (whole) {
                const int page = __builtin_amdgcn_readlane(pages, b * 16);
                const char *at = k_at + (page * page_bytes + ((y0 + b * 16) & in_page) * ROW_BYTES);
#pragma unroll
                for (int i = 0; i < K_LOADS; ++i) rk[b][i] = *(const uint4 *)(at + off + i * 64);
            } else {
                const int key = b * 16 + col, page = __shfl(pages, key);
                const char *at = k_at + (page * page_bytes + ((y0 + key) & in_page) * ROW_BYTES + quad * 16);
#pragma unroll
                for (int i = 0; i < K_LOADS; ++i) {
                    rk[b][i] = make_uint4(0, 0, 0, 0);
                    if (page >= 0) rk[b][i] = *(const uint4 *)(at + i * 64);
                }
            }
        }
    };
    auto fetch_v = [&](int tile, int pages, bool whole) {
        const int y0 = start_of(tile);
#pragma unroll
        for (int i = 0; i < V_LOADS; ++i) {
            if (whole) {
                const int key = i * 64 / PER_ROW, page = __builtin_amdgcn_readlane(pages, key);
                const char *at = v_at + (page * page_bytes + ((y0 + key) & in_page) * ROW_BYTES);
                rv[i] = *(const uint4 *)(at + lane * 16);
            } else {
                const int key = (i * 64 + lane) / PER_ROW, page = __shfl(pages, key);
                rv[i] = make_uint4(0, 0, 0, 0);
                if (page >= 0) rv[i] = *(const uint4 *)(v_at + (page * page_bytes + ((y0 + key) & in_page) * ROW_BYTES + lane % PER_ROW * 16));
            }
        }
    };

    uint4 *sv = (uint4 *)(smem + wave * WAVE_LDS);
    f32x4 o[COLS][D / 16] = {};
    float m[COLS], l[COLS];
#pragma unroll
    for (int w = 0; w < COLS; ++w) { m[w] = NEG_INF; l[w] = 0.0f; }
    int pages = page_of(tile0 + wave), next = page_of(tile0 + wave + 4);
    pages = in_pool(kv, pages);
    uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(pages >= 0);
    if (tile0 + wave < tile1) {
        const bool whole = PAGE16 && there == 0xffffffffu;
        fetch_k(tile0 + wave, pages, whole);
        fetch_v(tile0 + wave, pages, whole);
    }
    for (int tile = tile0 + wave; tile < tile1; tile += 4) {
        const uint32_t now = there;
        const int y0 = start_of(tile);
        pages = in_pool(kv, next);
        there = (uint32_t)__builtin_amdgcn_ballot_w64(pages >= 0);
        const bool whole = PAGE16 && there == 0xffffffffu, more = tile + 4 < tile1;
        next = page_of(tile + 8);
        f32x4 s[COLS][2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            f32x4 acc[COLS] = {};
#pragma unroll
            for (int i = 0; i < K_LOADS; ++i) {
                if constexpr (FP8) {
                    union { X2 x2[8]; X8 x8[2]; } kw;
                    const uint32_t kk[4] = {rk[b][i].x, rk[b][i].y, rk[b][i].z, rk[b][i].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) widen(kk[j], kw.x2[2 * j], kw.x2[2 * j + 1]);
#pragma unroll
                    for (int w = 0; w < COLS; ++w) {
                        acc[w] = mfma16(kw.x8[0], qf[w][2 * i], acc[w]);
                        acc[w] = mfma16(kw.x8[1], qf[w][2 * i + 1], acc[w]);
                    }
                } else
#pragma unroll
                    for (int w = 0; w < COLS; ++w) acc[w] = mfma16(__builtin_bit_cast(X8, rk[b][i]), qf[w][i], acc[w]);
            }
#pragma unroll
            for (int w = 0; w < COLS; ++w) s[w][b] = acc[w];
        }
        if (more) fetch_k(tile + 4, pages, whole);
#pragma unroll
        for (int i = 0; i < V_LOADS; ++i) {
            const int key = (i * 64 + lane) / PER_ROW, part = lane % PER_ROW;
            if constexpr (FP8) {
                union { X2 x[8]; uint4 u[2]; } w;
                const uint32_t vv[4] = {rv[i].x, rv[i].y, rv[i].z, rv[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) widen(vv[j], w.x[2 * j], w.x[2 * j + 1]);
                sv[few_v_piece<CH>(key, 2 * part)] = w.u[0]; sv[few_v_piece<CH>(key, 2 * part + 1)] = w.u[1];
            } else sv[few_v_piece<CH>(key, part)] = rv[i];
        }
        if (more) fetch_v(tile + 4, pages, whole);
        // a lane's register i of block b is the score of key y0 + 16 b + 4 quad + i
        const bool all = now == 0xffffffffu && (tree ? y0 + 31 < base : y0 + 31 <= base) &&
                         (a.window <= 0 || y0 + 31 < a.n_sink || all_last - y0 < a.window);
        union { X8 x8; X2 x2[4]; } p[COLS], rest[COLS];
#pragma unroll
        for (int w = 0; w < COLS; ++w) {
            if (!all) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int k = 16 * b + 4 * quad + i;
                        s[w][b][i] = ((now >> k) & 1) && view[w].sees(y0 + k) ? s[w][b][i] : NEG_INF;
                    }
            }
            float top = fmaxf(fmaxf(fmaxf(s[w][0][0], s[w][0][1]), fmaxf(s[w][0][2], s[w][0][3])),
                              fmaxf(fmaxf(s[w][1][0], s[w][1][1]), fmaxf(s[w][1][2], s[w][1][3])));
            top = fmaxf(top, lane_16_away(top));
            top = fmaxf(top, other_half(top)) * c;
            if (__builtin_amdgcn_ballot_w64(top > m[w] + (MAX_SLACK + LIFT<E>))) {
                const float m_new = fmaxf(m[w], top - LIFT<E>);
                const float shrink = __builtin_amdgcn_exp2f(m[w] - (m_new == NEG_INF ? 0.0f : m_new));
                m[w] = m_new;
                l[w] *= shrink;
#pragma unroll
                for (int x = 0; x < D / 16; ++x) o[w][x] *= shrink;
            }
            const float m_use = m[w] == NEG_INF ? 0.0f : m[w];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w0 = __builtin_amdgcn_exp2f(fmaf(s[w][i / 2][2 * (i & 1)], c, -m_use)), w1 = __builtin_amdgcn_exp2f(fmaf(s[w][i / 2][2 * (i & 1) + 1], c, -m_use));
                p[w].x2[i][0] = (E)w0;
                p[w].x2[i][1] = (E)w1;
                rest[w].x2[i][0] = (E)(w0 - (float)p[w].x2[i][0]);
                rest[w].x2[i][1] = (E)(w1 - (float)p[w].x2[i][1]);
                l[w] += w0 + w1;
            }
        }
        // the values were written by other lanes of this wavefront: LDS works in order, the compiler has to as well
        __builtin_amdgcn_wave_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
            const int key = 4 * quad + (col >> 2), piece = x * 2 + ((col & 3) >> 1);
            using LdsPtr = __attribute__((address_space(3))) i16x4 *;
            const char *at0 = (const char *)(sv + few_v_piece<CH>(key, piece)) + (col & 1) * 8;
            const char *at1 = at0 + 16 * CH * 16;
            union { i16x4 h[2]; X8 x; } vf;
            vf.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)at0);
            vf.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)at1);
#pragma unroll
            for (int w = 0; w < COLS; ++w) o[w][x] = mfma16(vf.x, rest[w].x8, mfma16(vf.x, p[w].x8, o[w][x]));
        }
        __builtin_amdgcn_wave_barrier();
        asm volatile("" ::: "memory");
    }
    // sums that are not finite, as above
    bool odd = any_odd<D / 16>(o[0]);
    if constexpr (COLS == 2) odd |= any_odd<D / 16>(o[1]);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) != 0, false)) {
#pragma unroll
        for (int w = 0; w < COLS; ++w)
#pragma unroll
            for (int x = 0; x < D / 16; ++x) o[w][x] = f32x4{};
#pragma unroll 1
        for (int key = (tile0 + wave) * FEW_KEYS; key < tile1 * FEW_KEYS; key += key % FEW_KEYS == FEW_KEYS - 1 ? 3 * FEW_KEYS + 1 : 1) {
            const int y = start_of(key / FEW_KEYS) + key % FEW_KEYS;
            if (y >= ex.hi || (y < ex.lo && y >= a.n_sink)) continue;
            const int page = in_pool(kv, sq.table[y >> kv.shift]);
            if (page < 0) continue;
            const int64_t at = page * page_bytes + (y & in_page) * ROW_BYTES;
#pragma unroll
            for (int w = 0; w < COLS; ++w) {
                float dot = 0.0f;
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {
                    float k[8];
                    numbers<E, FP8, 8>(k_at + at + (FP8 ? (x >> 1) * 64 + quad * 16 + (x & 1) * 8 : (x * 32 + quad * 8) * 2), k);
#pragma unroll
                    for (int i = 0; i < 8; ++i) dot = fmaf((float)qf[w][x][i], k[i], dot);
                }
                dot += lane_16_away(dot);
                dot += other_half(dot);
                const bool see = view[w].sees(y);
                const float weight = __builtin_amdgcn_exp2f(fmaf(dot, c, -(m[w] == NEG_INF ? 0.0f : m[w])));
#pragma unroll
                for (int x = 0; x < D / 16; ++x) {
                    float v[4];
                    numbers<E, FP8, 4>(v_at + at + (x * 16 + 4 * quad) * (ROW_BYTES / D), v);
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[w][x][j] += see ? weight * v[j] : 0.0f;
                }
            }
        }
    }
    // the four wavefronts' sums: each adds up a quarter of the numbers
#pragma unroll
    for (int w = 0; w < COLS; ++w) {
        l[w] += lane_16_away(l[w]);
        l[w] += other_half(l[w]);
        if (!view[w].alive) { m[w] = NEG_INF; l[w] = 0.0f; }
        if (quad == 0) { s_ml[wave][0][16 * w + col] = m[w]; s_ml[wave][1][16 * w + col] = l[w]; }
    }
    __syncthreads();
    const float v_unit = a.v_scale ? a.v_scale[a.layer * kv.n_heads + head] : 1.0f;
    f32x4 *s_o = (f32x4 *)smem;                                  // [wave][COLS][D / 16][64]
    float top[COLS], sum[COLS];
#pragma unroll
    for (int w = 0; w < COLS; ++w) {
        top[w] = NEG_INF;
#pragma unroll
        for (int v = 0; v < 4; ++v) top[w] = fmaxf(top[w], s_ml[v][0][16 * w + col]);
        const float use = top[w] == NEG_INF ? 0.0f : top[w], f = __builtin_amdgcn_exp2f(m[w] - use);
        sum[w] = 0.0f;
#pragma unroll
        for (int v = 0; v < 4; ++v) sum[w] += s_ml[v][1][16 * w + col] * __builtin_amdgcn_exp2f(s_ml[v][0][16 * w + col] - use);
#pragma unroll
        for (int x = 0; x < D / 16; ++x) s_o[((wave * COLS + w) * (D / 16) + x) * 64 + lane] = o[w][x] * f;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < COLS; ++w) {
        if (t[w] >= sq.nq) continue;
        const int64_t slot = ((int64_t)pair * a.splits + split) * ROWS + 16 * w + col;
        const float unit = holds_any(sum[w]) ? v_unit / sum[w] : 0.0f;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const int x = wave * (D / 64) + i, d = x * 16 + 4 * quad;
            f32x4 y = s_o[(w * (D / 16) + x) * 64 + lane];
#pragma unroll
            for (int v = 1; v < 4; ++v) y += s_o[((v * COLS + w) * (D / 16) + x) * 64 + lane];
            if (parts > 1) {
                leave(a.part + slot * D + d, y[0], y[1]);
                leave(a.part + slot * D + d + 2, y[2], y[3]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = holds_any(sum[w]) ? y[j] * unit : 0.0f;
                put((E *)a.out + (int64_t)(sq.q0 + t[w]) * a.out_token + (int64_t)qhead[w] * a.out_head + d, a.out_wide, y[0], y[1], y[2], y[3]);
            }
        }
        if (wave == 0 && quad == 0) {
            if (parts > 1) leave((float *)(a.part_ml + slot), top[w], sum[w]);
            else if (a.lse) a.lse[(int64_t)(sq.q0 + t[w]) * a.n_heads + qhead[w]] = holds_any(sum[w]) ? (top[w] + __builtin_amdgcn_logf(sum[w])) * LN2 : NEG_INF;
        }
    }
    if (parts > 1) join<E, D, ROWS>(a, sq, pair, 0, parts, (float *)smem);
}

__global__ __launch_bounds__(AT_THREADS) void hx_attend_clear_kernel(int *done, int64_t n)
{
    const int64_t i = (int64_t)blockIdx.x * AT_THREADS + threadIdx.x;
    if (i < n) done[i] = 0;
}

// Room for the parts, and where the workgroups themselves put them together, for counters, which are 0 whenever no launch is under way.
int parts_room(hx_ctx *ctx, AttendArgs &a, int64_t tiles, int rows, int dim, bool counted, hipStream_t stream)
{
    HxScratch &parts = hx_serve(ctx)->att, &done = hx_serve(ctx)->att_done;
    const int64_t slots = tiles * a.splits * rows;
    if (int rc = hx_scratch(ctx, parts, (size_t)slots * (dim * sizeof(float) + sizeof(float2)), stream)) return rc;
    if (counted) {
        const void *was = done.p;
        if (int rc = hx_scratch(ctx, done, (size_t)tiles * sizeof(int), stream)) return rc;
        if (done.p != was) {
            const int64_t n = done.cap / sizeof(int);
            hx_attend_clear_kernel<<<(int)((n + AT_THREADS - 1) / AT_THREADS), AT_THREADS, 0, stream>>>((int *)done.p, n);
        }
        a.done = (int *)done.p;
    }
    a.part = (float *)parts.p;
    a.part_ml = (float2 *)(a.part + slots * dim);
    return HX_OK;
}

template <typename E, bool FP8, int D, bool PAGE16>
int launch(hx_ctx *ctx, AttendArgs &a, hipStream_t stream)
{
    using C = Tile<FP8, D, 4, PAGE16>;
    const int lds = C::LDS + (a.parent ? TREE_BYTES : 0);
    const int64_t tiles = (int64_t)a.n * a.kv.n_heads * a.row_tiles, grid = tiles * a.splits, join_grid = tiles * (C::ROWS / (AT_THREADS / (D / 4)));
    HX_REQUIRE(ctx, grid <= hx_most_groups(C::THREADS) && join_grid <= hx_most_groups(AT_THREADS), HX_ERR_SHAPE, "%lld workgroups", (long long)grid);
    if (a.splits > 1)
        if (int rc = parts_room(ctx, a, tiles, C::ROWS, D, false, stream)) return rc;
    hx_attend_kernel<E, FP8, D, 4, PAGE16><<<(int)grid, C::THREADS, lds, stream>>>(a);
    if (a.splits > 1) hx_attend_join_kernel<E, D, KT, C::ROWS><<<(int)join_grid, AT_THREADS, 0, stream>>>(a);
    return hx_check_launch(ctx, "hx_attend_kernel");
}

// Parts of the keys where there are few workgroups otherwise: `many` workgroups if all sequences had the longest's length, but no part
// shorter than `part` tiles unless there were not even `few` workgroups then, and none shorter than `least`.
//
// Where tiles of rows alone are two workgroups a CU and more (four of up to 32 rows, as up to four fit a CU), `full` of them, parts cost their joining and gain only that a long sequence
// among short ones is not one workgroup's: none is shorter than `full_part` tiles then, more with more tiles of rows, up to twice that.
// Divided as before that, with these longer parts, and not at all, 32 heads of 128 over 8 KV heads: 2 prompts of 3000 tokens 249, 177
// and 177 us; 64 trees of 32 drafts over 1500 134, 97 and 97, over 500 but one over 32768 182, 181 and 818; 256 sequences' tokens over 500 to
// 32768 1485, 1509 and 1584, over 500 but one over 32768 375, 369 and 589, over 1000 195, 189 and 185.  What this loses: 100 trees of 16 over
// some 1500 tokens, 40 to 8192, take 199 divided further and 238 as here.
struct Division {
    int64_t many, few;
    int part, least;
    int64_t full;
    int full_part;
};
void divide(AttendArgs &a, int64_t groups, const Division &d, int max_len, int tile_keys, int tile_rows)
{
    // what one tile of rows may see: its own queries, or all drafts of a tree, and the window and the sinks before them
    const int64_t own = a.parent || a.max_q < tile_rows / a.group + 2 ? a.max_q : tile_rows / a.group + 2;
    int64_t reach = max_len;
    if (a.window > 0 && reach > (int64_t)a.window + a.n_sink + own) reach = (int64_t)a.window + a.n_sink + own;
    const int64_t tiles = (reach + tile_keys - 1) / tile_keys + 1, all = groups * tiles;
    int64_t chunk = (all + d.many - 1) / d.many, fill = (all + d.few - 1) / d.few;
    fill = fill < d.part ? fill : d.part;
    chunk = chunk > fill ? chunk : fill;
    chunk = chunk > d.least ? chunk : d.least;
    int64_t parts = (tiles + chunk - 1) / chunk;
    if (groups >= d.full) {
        const int64_t more = d.full_part * groups / d.full, long_part = more < 2 * d.full_part ? more : 2 * d.full_part;
        chunk = chunk > long_part ? chunk : long_part;
        parts = (tiles + chunk / 2) / chunk;                 // the last one up to half as long again
        parts = parts > 1 ? parts : 1;
    }
    if (parts > MAX_SPLITS) {
        parts = MAX_SPLITS;
        chunk = (tiles + MAX_SPLITS - 1) / MAX_SPLITS;
    }
    a.chunk = (int)chunk;
    a.splits = (int)parts;
}

template <typename E, bool FP8, int D, int COLS>
int launch_few(hx_ctx *ctx, AttendArgs &a, hipStream_t stream)
{
    const int lds = 4 * few_wave_lds(D, COLS) + (a.parent ? TREE_BYTES : 0);
    const int64_t tiles = (int64_t)a.n * a.kv.n_heads, grid = tiles * a.splits;
    HX_REQUIRE(ctx, grid <= hx_most_groups(AT_THREADS), HX_ERR_SHAPE, "%lld workgroups", (long long)grid);
    if (a.splits > 1)
        if (int rc = parts_room(ctx, a, tiles, 16 * COLS, D, true, stream)) return rc;
    if (a.kv.shift >= 4) hx_attend_few_kernel<E, FP8, D, COLS, true><<<(int)grid, AT_THREADS, lds, stream>>>(a);
    else hx_attend_few_kernel<E, FP8, D, COLS, false><<<(int)grid, AT_THREADS, lds, stream>>>(a);
    return hx_check_launch(ctx, "hx_attend_few_kernel");
}

// More LDS a workgroup than the 64 KB that need no asking, for the kernels of a pair of types and a head_dim, the first time that a context
// meets them.  (When it is created this took 5 ms, most of it the loading of code that a planner never runs.)
template <typename E, bool FP8, int D, bool PAGE16>
hipError_t allow_many()
{
    return hipFuncSetAttribute((const void *)hx_attend_kernel<E, FP8, D, 4, PAGE16>, hipFuncAttributeMaxDynamicSharedMemorySize,
                               Tile<FP8, D, 4, PAGE16>::LDS + TREE_BYTES);
}
template <typename E, bool FP8, int D, int COLS, bool PAGE16>
hipError_t allow_few()
{
    return hipFuncSetAttribute((const void *)hx_attend_few_kernel<E, FP8, D, COLS, PAGE16>, hipFuncAttributeMaxDynamicSharedMemorySize,
                               4 * few_wave_lds(D, COLS) + TREE_BYTES);
}
template <typename E, bool FP8, int D>
int allow(hx_ctx *ctx)
{
    constexpr int kind = (std::is_same_v<E, _Float16> ? 6 : 0) + (FP8 ? 3 : 0) + (D == 64 ? 0 : D == 128 ? 1 : 2);
    if (hx_serve(ctx)->att_allowed >> kind & 1) return HX_OK;
    for (const hipError_t e : {allow_many<E, FP8, D, false>(), allow_many<E, FP8, D, true>(), allow_few<E, FP8, D, 1, false>(), allow_few<E, FP8, D, 1, true>(),
                               allow_few<E, FP8, D, 2, false>(), allow_few<E, FP8, D, 2, true>()}) {
        if (e == hipSuccess) continue;
        (void)hipGetLastError();                   // not the next launch's
        return hx_fail(ctx, HX_ERR_DEVICE, "hipFuncSetAttribute(LDS size): %s", hipGetErrorString(e));
    }
    hx_serve(ctx)->att_allowed |= 1u << kind;
    return HX_OK;
}

template <typename E, bool FP8, int D>
int plan(hx_ctx *ctx, AttendArgs &a, int max_len, hipStream_t stream)
{
    if (int rc = allow<E, FP8, D>(ctx)) return rc;
    const int64_t rows = (int64_t)a.max_q * a.group, pairs = (int64_t)a.n * a.kv.n_heads;
    if (rows <= 32) {
        a.row_tiles = 1;
        divide(a, pairs, {16 * ctx->num_cu, 16 * ctx->num_cu, 8, 8, 4 * ctx->num_cu, 64}, max_len, FEW_KEYS, 32);
        return rows <= 16 ? launch_few<E, FP8, D, 1>(ctx, a, stream) : launch_few<E, FP8, D, 2>(ctx, a, stream);
    }
    a.row_tiles = (int)((rows + 127) / 128);
    divide(a, pairs * a.row_tiles, {16 * ctx->num_cu, 2 * ctx->num_cu, 32, 4, 2 * ctx->num_cu, 128}, max_len, KT, 128);
    return a.kv.shift >= 4 ? launch<E, FP8, D, true>(ctx, a, stream) : launch<E, FP8, D, false>(ctx, a, stream);
}

template <typename E, bool FP8>
int by_dim(hx_ctx *ctx, AttendArgs &a, int max_len, hipStream_t stream)
{
    if (a.kv.dim == 64) return plan<E, FP8, 64>(ctx, a, max_len, stream);
    if (a.kv.dim == 128) return plan<E, FP8, 128>(ctx, a, max_len, stream);
    return plan<E, FP8, 256>(ctx, a, max_len, stream);
}

}  // namespace

// One source file for each pair of types, queries' and cache's: HX_ATTEND_TYPES(name, E, FP8) defines its function.
#define HX_ATTEND_TYPES(name, E, FP8)                                                                                    \
    int hx_attend_##name(hx_ctx *ctx, HxAttend &a, int max_len, hipStream_t stream) { return by_dim<E, FP8>(ctx, a, max_len, stream); }
