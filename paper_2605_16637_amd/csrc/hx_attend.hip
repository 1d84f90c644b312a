// Attention of a few or many queries over cached pages: sliding windows with sinks, trees of drafted tokens.
//
// One pass over the keys with a running maximum and sum.  The products are taken transposed, S^T = K Q^T and O^T = V^T P^T: a
// lane then holds one query's scores, its maximum needs one exchange between the two halves of the wavefront, the running
// maximum scales a lane's own accumulators, and the weights leave the first product in the very registers that the second wants them
// in (the order in which keys are summed is free, so the second product takes them in the first's order and the
// values are read from LDS in that order, transposed on the way).
#include "hx_serve.hpp"

#include <type_traits>

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

template <typename E> struct Types;
template <> struct Types<__bf16> { using x8 = bf16x8; using x4 = bf16x4; using x2 = bf16x2; };
template <> struct Types<_Float16> { using x8 = f16x8; using x4 = f16x4; using x2 = f16x2; };

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
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

struct AttendArgs {
    KvView kv;
    int layer, n;
    const int32_t *row, *q_ptr;
    int n_q, max_q, n_heads, group;
    const void *q;
    int64_t q_token, q_head;
    void *out;
    int64_t out_token, out_head;
    float *lse;
    float scale;
    int window, n_sink;
    const int32_t *parent;
    const float *k_scale, *v_scale;
    bool q_wide, out_wide;       // q can be read 16 bytes at a time, out written 8
    int row_tiles, splits;
    float *part;                 // [workgroup][rows][dim], when splits > 1
    float2 *part_ml;             // [workgroup][rows] maximum (of s log2 e) and sum
};

constexpr int AT_THREADS = 256;

// one value of the other half of the wavefront
__device__ __forceinline__ float other_half(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}

// WR wavefronts beside each other take 32 rows each (a row: one query and query head of the KV head), 4 / WR share a tile's keys.
template <typename E, bool FP8, int D, int WR>
struct Tile {
    static constexpr int WK = 4 / WR;
    static constexpr int NK = WR == 4 ? 2 : 1;           // blocks of 32 keys a wavefront takes of a tile
    static constexpr int KT = WK * NK * 32;              // keys of a tile
    static constexpr int ROWS = 32 * WR;
    static constexpr int CH = D / 8;                     // 16-byte pieces of a row in LDS
    static constexpr int LOADS = KT * CH / AT_THREADS / (FP8 ? 2 : 1);   // of a thread, 16 bytes each, keys or values
    static constexpr int LDS = 2 * KT * D * 2;
    // the drafts' tree: depth of each, and the bits of those above each row's query
    static constexpr int TREE = HX_MAX_DRAFTS * 4 + HX_MAX_DRAFTS * (HX_MAX_DRAFTS / 32) * 4;
};

// Where 16-byte piece c of key row r lies in LDS.  Keys are read 32 rows at a time at one piece; the pieces of 8 rows and more fall in
// different banks.  Values are read as 4 rows x 64 bytes; those rows' pieces, too.
template <int CH> __device__ __forceinline__ int k_piece(int r, int c) { return r * CH + (c ^ (r & (CH < 16 ? CH - 1 : 15))); }
template <int CH> __device__ __forceinline__ int v_piece(int r, int c) { return r * CH + (c ^ (CH >= 16 ? (r & 3) << 2 : ((r >> 1) & 1) << 2)); }

template <typename E, bool FP8, int D, int WR>
__global__ __launch_bounds__(AT_THREADS, D == 256 ? 1 : 2) void hx_attend_kernel(AttendArgs a)
{
    using X8 = typename Types<E>::x8;
    using X4 = typename Types<E>::x4;
    using X2 = typename Types<E>::x2;
    using C = Tile<E, FP8, D, WR>;
    constexpr int KT = C::KT, CH = C::CH, LOADS = C::LOADS, NK = C::NK, WK = C::WK;
    extern __shared__ __align__(16) char smem[];
    uint4 *sk = (uint4 *)smem, *sv = sk + KT * CH;
    int *s_depth = (int *)(smem + C::LDS);
    uint32_t *s_anc = (uint32_t *)(s_depth + HX_MAX_DRAFTS);     // [HX_MAX_DRAFTS][HX_MAX_DRAFTS / 32]
    __shared__ float s_ml[4][2][32];

    const KvView &kv = a.kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, col = lane & 31;
    const int wr = wave % WR, wk = wave / WR;
    const int nh = a.n * kv.n_heads;
    const int pair = blockIdx.x % nh, rest = blockIdx.x / nh;
    const int split = rest % a.splits, rt = a.row_tiles - 1 - rest / a.splits;
    const int seq = pair / kv.n_heads, head = pair % kv.n_heads;

    // the sequence and its queries
    const int q0 = a.q_ptr[seq], q1 = a.q_ptr[seq + 1], nq = q1 - q0, r = a.row ? a.row[seq] : seq;
    if (q0 < 0 || nq < 0 || q1 > a.n_q) { if (tid == 0) hx_raise(kv.status, HX_ERR_INDEX); return; }
    if (rt * C::ROWS >= nq * (int64_t)a.group) return;
    bool ok = r >= 0 && r < kv.rows && nq <= a.max_q;
    const int len = ok ? kv.len[r] : 0;
    ok = ok && hx_row_ok(kv, r, len) && nq <= len;
    if (!ok && tid == 0) hx_raise(kv.status, HX_ERR_INDEX);
    const int base = len - nq;
    const int32_t *table = hx_row(kv, ok ? r : 0);

    const bool tree = a.parent != nullptr;
    if (tree && ok) {
        // every draft's depth and the drafts above it
        int *s_parent = (int *)smem;
        if (tid < nq) s_parent[tid] = a.parent[q0 + tid];
        __syncthreads();
        if (tid < nq) {
            uint32_t *mine = s_anc + tid * (HX_MAX_DRAFTS / 32);
            for (int w = 0; w < HX_MAX_DRAFTS / 32; ++w) mine[w] = 0;
            int depth = 0, at = tid;
            while (at >= 0) {
                mine[at >> 5] |= 1u << (at & 31);
                const int up = s_parent[at];
                if (up >= at || up < -2) { hx_raise(kv.status, HX_ERR_INDEX); at = -2; break; }
                at = up;
                ++depth;
            }
            s_depth[tid] = at == -2 ? -1 : depth - 1;          // -1: left out
        }
        __syncthreads();
    }

    // this lane's row
    const int row = rt * C::ROWS + wr * 32 + col, t = row / a.group, e = row % a.group;
    bool alive = ok && t < nq;
    int pos = base + t;
    if (tree && alive) {
        alive = s_depth[t] >= 0;
        pos = base + s_depth[t];
    }
    const int qhead = head * a.group + e;

    const float k_unit = a.k_scale ? a.k_scale[a.layer * kv.n_heads + head] : 1.0f;
    const float sc = a.scale * k_unit * LOG2E;
    // the score's sign goes into the query, and its factor is no 0: a masked score stays -infinity
    const float c = fmaxf(fabsf(sc), 1e-37f);
    X8 qf[D / 16];
    {
        const E *qp = (const E *)a.q + (int64_t)(q0 + t) * a.q_token + (int64_t)qhead * a.q_head;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            X8 x = {};
            if (alive) {
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

    // the keys that some row of this tile of rows may see: the sinks below `sink_end`, then lo .. hi-1
    int hi = 0, lo = 0;
    const int t_first = (int)((int64_t)rt * C::ROWS / a.group);
    int t_last = (int)(((int64_t)rt * C::ROWS + C::ROWS - 1) / a.group);
    t_last = t_last < nq ? t_last : nq - 1;
    if (ok) {
        hi = tree ? len : base + t_last + 1;
        if (a.window > 0) {
            const int first_pos = tree ? base - 1 : base + t_first;         // the least position of a query
            lo = first_pos - a.window + 1;
            lo = lo > 0 ? lo : 0;
            if (tree && lo > base) lo = base;
        }
    }
    int sink_tiles = 0, lo_tile = lo / KT;
    if (a.window > 0 && lo > 0) {
        const int sinks = a.n_sink < lo ? a.n_sink : lo;
        sink_tiles = (sinks + KT - 1) / KT;
        if (sink_tiles >= lo_tile) { sink_tiles = 0; lo_tile = 0; }
    }
    const int tiles = sink_tiles + (hi + KT - 1) / KT - lo_tile;
    const int n_tiles = hi > 0 ? tiles : 0;
    const int tile0 = (int)((int64_t)n_tiles * split / a.splits), tile1 = (int)((int64_t)n_tiles * (split + 1) / a.splits);

    // rows of this wavefront: between which positions they lie (for a tile that all of them see whole)
    int wave_first = base + (rt * C::ROWS + wr * 32) / a.group, wave_last = base + (rt * C::ROWS + wr * 32 + 31) / a.group;
    if (tree) { wave_first = base - 1; wave_last = len; }

    constexpr int KEYS_LANE = (KT + 63) / 64;
    auto start_of = [&](int tile) { return (tile < sink_tiles ? tile : tile - sink_tiles + lo_tile) * KT; };
    // the page of the key that lane l stands for, -1 where there is nothing to see
    auto page_of = [&](int tile, int j) {
        const int y = start_of(tile) + j * 64 + lane;
        int page = -1;
        if (tile < tile1 && (KT >= 64 || lane < KT) && y < hi && (y >= lo || y < a.n_sink)) page = table[y >> kv.shift];
        if (page >= kv.n_pages) { hx_raise(kv.status, HX_ERR_INDEX); page = -1; }
        return page;
    };

    uint4 rk[LOADS], rv[LOADS];
    int pages[KEYS_LANE];
    const int64_t layer_at = (int64_t)a.layer * kv.n_pages;
    constexpr int ROW_BYTES = FP8 ? D : 2 * D, PER_ROW = ROW_BYTES / 16;
    auto fetch = [&](int tile) {
        const int y0 = start_of(tile);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int piece = i * AT_THREADS + tid, key = piece / PER_ROW, part = piece % PER_ROW;
            const int page = __shfl(pages[KEYS_LANE > 1 ? (i * AT_THREADS) / PER_ROW / 64 : 0], key & 63);
            const int tok = (y0 + key) & ((1 << kv.shift) - 1);
            const int64_t at = ((((layer_at + page) * kv.n_heads + head) << kv.shift) + tok) * ROW_BYTES + part * 16;
            rk[i] = rv[i] = make_uint4(0, 0, 0, 0);
            if (page >= 0) {
                rk[i] = *(const uint4 *)((const char *)kv.k + at);
                rv[i] = *(const uint4 *)((const char *)kv.v + at);
            }
        }
    };
    auto store = [&]() {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int piece = i * AT_THREADS + tid, key = piece / PER_ROW, part = piece % PER_ROW;
            if constexpr (FP8) {
                union { X2 x[8]; uint4 u[2]; } wk_, wv_;
                const uint32_t kk[4] = {rk[i].x, rk[i].y, rk[i].z, rk[i].w}, vv[4] = {rv[i].x, rv[i].y, rv[i].z, rv[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) { widen(kk[j], wk_.x[2 * j], wk_.x[2 * j + 1]); widen(vv[j], wv_.x[2 * j], wv_.x[2 * j + 1]); }
                sk[k_piece<CH>(key, 2 * part)] = wk_.u[0]; sk[k_piece<CH>(key, 2 * part + 1)] = wk_.u[1];
                sv[v_piece<CH>(key, 2 * part)] = wv_.u[0]; sv[v_piece<CH>(key, 2 * part + 1)] = wv_.u[1];
            } else {
                sk[k_piece<CH>(key, part)] = rk[i];
                sv[v_piece<CH>(key, part)] = rv[i];
            }
        }
    };

    f32x16 o[D / 32] = {};
    float m = NEG_INF, l = 0.0f;

#pragma unroll
    for (int j = 0; j < KEYS_LANE; ++j) pages[j] = page_of(tile0, j);
    if (tile0 < tile1) fetch(tile0);
    for (int tile = tile0; tile < tile1; ++tile) {
        unsigned long long there[KEYS_LANE];
#pragma unroll
        for (int j = 0; j < KEYS_LANE; ++j) {
            there[j] = __builtin_amdgcn_ballot_w64(pages[j] >= 0);
            pages[j] = page_of(tile + 1, j);
        }
        __syncthreads();
        store();
        __syncthreads();
        if (tile + 1 < tile1) fetch(tile + 1);

        const int y0 = start_of(tile);
        f32x16 s[NK];
#pragma unroll
        for (int b = 0; b < NK; ++b) {
            const int key = (wk * NK + b) * 32 + col;
            f32x16 acc = {};
#pragma unroll
            for (int x = 0; x < D / 16; ++x) {
                const uint4 kf = sk[k_piece<CH>(key, 2 * x + half)];
                acc = mfma32(__builtin_bit_cast(X8, kf), qf[x], acc);
            }
            s[b] = acc;
        }
        // a lane's register i of block b is the score of key y0 + (wk NK + b) 32 + 8 (i / 4) + 4 half + i % 4
#pragma unroll
        for (int b = 0; b < NK; ++b) {
            const int blk = (wk * NK + b) * 32, yb = y0 + blk;
            const uint32_t seen = (uint32_t)(there[blk / 64] >> (blk & 32));
            const bool all = seen == 0xffffffffu && (tree ? yb + 31 < base : yb + 31 <= wave_first) &&
                             (a.window <= 0 || yb + 31 < a.n_sink || wave_last - yb < a.window);
            if (!all) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int k = 8 * (i / 4) + 4 * half + i % 4, y = yb + k;
                    bool see = alive && ((seen >> k) & 1);
                    int ypos = y;
                    if (tree && y >= base) {
                        const int d = y - base;
                        const bool in = d < nq;
                        see = see && in && ((s_anc[(t < nq ? t : 0) * (HX_MAX_DRAFTS / 32) + ((in ? d : 0) >> 5)] >> (d & 31)) & 1);
                        ypos = base + s_depth[in ? d : 0];
                    }
                    see = see && ypos <= pos && (a.window <= 0 || ypos < a.n_sink || pos - ypos < a.window);
                    s[b][i] = see ? s[b][i] : NEG_INF;
                }
            }
        }
        float top = NEG_INF;
#pragma unroll
        for (int b = 0; b < NK; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        top = fmaxf(top, other_half(top)) * c;
        const float m_new = fmaxf(m, top), m_use = m_new == NEG_INF ? 0.0f : m_new;
        const float shrink = __builtin_amdgcn_exp2f(m - m_use);
        m = m_new;
        l *= shrink;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) o[x] *= shrink;
#pragma unroll
        for (int b = 0; b < NK; ++b) {
            X8 p[2];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float w = __builtin_amdgcn_exp2f(fmaf(s[b][i], c, -m_use));
                l += w;
                p[i / 8][i % 8] = (E)w;
            }
            const int blk = (wk * NK + b) * 32;
#pragma unroll
            for (int st = 0; st < 2; ++st) {
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {
                    // 4 keys x 16 numbers a group of 16 lanes: its lane j reads 4 numbers of key j / 4 and gets number j of the 4 keys
                    const int g16 = (lane >> 4) & 1, j = lane & 15;
                    const int key = blk + st * 16 + 4 * half + (j >> 2), piece = x * 4 + g16 * 2 + ((j & 3) >> 1);
                    using LdsPtr = __attribute__((address_space(3))) i16x4 *;
                    const char *at0 = (const char *)(sv + v_piece<CH>(key, piece)) + (j & 1) * 8;
                    const char *at1 = (const char *)(sv + v_piece<CH>(key + 8, piece)) + (j & 1) * 8;
                    union { i16x4 h[2]; X8 x; } vf;
                    vf.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)at0);
                    vf.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)at1);
                    o[x] = mfma32(vf.x, p[st], o[x]);
                }
            }
        }
    }

    l += other_half(l);
    if (!alive) { m = NEG_INF; l = 0.0f; }
    if constexpr (WK > 1) {
        // the wavefronts that shared the keys: common maximum, then the first of them adds the others' sums up
        if (half == 0) { s_ml[wave][0][col] = m; s_ml[wave][1][col] = l; }
        __syncthreads();
        float top = NEG_INF;
#pragma unroll
        for (int w = 0; w < WK; ++w) top = fmaxf(top, s_ml[w * WR + wr][0][col]);
        const float use = top == NEG_INF ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WK; ++w) sum += s_ml[w * WR + wr][1][col] * __builtin_amdgcn_exp2f(s_ml[w * WR + wr][0][col] - use);
        const float f = __builtin_amdgcn_exp2f(m - use);
        float *s_o = (float *)smem;
        if (wk > 0)
#pragma unroll
            for (int x = 0; x < D / 32; ++x)
#pragma unroll
                for (int i = 0; i < 16; ++i) s_o[(((wk - 1) * WR + wr) * (D / 2) + x * 16 + i) * 64 + lane] = o[x][i] * f;
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float y = o[x][i] * f;
#pragma unroll
                for (int w = 0; w < WK - 1; ++w) y += s_o[((w * WR + wr) * (D / 2) + x * 16 + i) * 64 + lane];
                o[x][i] = y;
            }
        m = top;
        l = sum;
    }
    if (t >= nq) return;
    if (a.splits > 1) {
        const int64_t slot = (((int64_t)pair * a.row_tiles + rt) * a.splits + split) * C::ROWS + wr * 32 + col;
        float *to = a.part + slot * D;
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 y = make_float4(o[x][4 * i], o[x][4 * i + 1], o[x][4 * i + 2], o[x][4 * i + 3]);
                *(float4 *)(to + x * 32 + 8 * i + 4 * half) = y;
            }
        if (half == 0) a.part_ml[slot] = make_float2(m, l);
        return;
    }
    const float v_unit = a.v_scale ? a.v_scale[a.layer * kv.n_heads + head] : 1.0f;
    const float f = l > 0.0f ? v_unit / l : 0.0f;
    E *to = (E *)a.out + (int64_t)(q0 + t) * a.out_token + (int64_t)qhead * a.out_head;
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            X4 y;
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = l > 0.0f ? (E)(o[x][4 * i + j] * f) : (E)0.0f;
            E *at = to + x * 32 + 8 * i + 4 * half;
            if (a.out_wide) *(X4 *)at = y;
            else
#pragma unroll
                for (int j = 0; j < 4; ++j) at[j] = y[j];
        }
    if (a.lse && half == 0) a.lse[(int64_t)(q0 + t) * a.n_heads + qhead] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * LN2 : NEG_INF;
}

// The parts of a row's keys put together: 4 numbers a thread.
template <typename E>
__global__ __launch_bounds__(AT_THREADS) void hx_attend_join_kernel(AttendArgs a, int rows)
{
    using X4 = typename Types<E>::x4;
    const KvView &kv = a.kv;
    const int per = kv.dim / 4;
    const int64_t u = (int64_t)blockIdx.x * AT_THREADS + threadIdx.x;
    const int d = (int)(u % per) * 4;
    const int64_t all_rows = (int64_t)a.max_q * a.group, pr = u / per;
    const int row = (int)(pr % all_rows);
    const int64_t pair = pr / all_rows;
    if (pair >= (int64_t)a.n * kv.n_heads) return;
    const int seq = (int)(pair / kv.n_heads), head = (int)(pair % kv.n_heads);
    const int q0 = a.q_ptr[seq], q1 = a.q_ptr[seq + 1], t = row / a.group, e = row % a.group;
    if (q0 < 0 || q1 > a.n_q || t >= q1 - q0) return;
    const int64_t slot0 = ((pair * a.row_tiles + row / rows) * a.splits) * rows + row % rows;
    float top = NEG_INF;
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, a.part_ml[slot0 + (int64_t)s * rows].x);
    const float use = top == NEG_INF ? 0.0f : top;
    float l = 0.0f;
    float4 o = make_float4(0, 0, 0, 0);
    for (int s = 0; s < a.splits; ++s) {
        const int64_t slot = slot0 + (int64_t)s * rows;
        const float2 ml = a.part_ml[slot];
        const float4 x = *(const float4 *)(a.part + slot * kv.dim + d);
        const float f = __builtin_amdgcn_exp2f(ml.x - use);
        if (ml.y > 0.0f) { l += ml.y * f; o.x += x.x * f; o.y += x.y * f; o.z += x.z * f; o.w += x.w * f; }
    }
    const float v_unit = a.v_scale ? a.v_scale[a.layer * kv.n_heads + head] : 1.0f;
    const float f = l > 0.0f ? v_unit / l : 0.0f;
    const int qhead = head * a.group + e;
    E *to = (E *)a.out + (int64_t)(q0 + t) * a.out_token + (int64_t)qhead * a.out_head + d;
    X4 y;
    y[0] = (E)(o.x * f); y[1] = (E)(o.y * f); y[2] = (E)(o.z * f); y[3] = (E)(o.w * f);
    if (a.out_wide) *(X4 *)to = y;
    else
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = y[j];
    if (a.lse && d == 0) a.lse[(int64_t)(q0 + t) * a.n_heads + qhead] = l > 0.0f ? (top + __builtin_amdgcn_logf(l)) * LN2 : NEG_INF;
}

template <typename E, bool FP8, int D, int WR>
int launch(hx_ctx *ctx, AttendArgs &a, hipStream_t stream)
{
    using C = Tile<E, FP8, D, WR>;
    const int lds = C::LDS + (a.parent ? C::TREE : 0);
    const int64_t grid = (int64_t)a.n * a.kv.n_heads * a.row_tiles * a.splits;
    HX_REQUIRE(ctx, grid <= INT32_MAX, HX_ERR_SHAPE, "%lld workgroups", (long long)grid);
    if (a.splits > 1) {
        const size_t slots = (size_t)grid * C::ROWS;
        if (int rc = hx_scratch(ctx, ctx->att, slots * (D * sizeof(float) + sizeof(float2)))) return rc;
        a.part = (float *)ctx->att.p;
        a.part_ml = (float2 *)(a.part + slots * D);
    }
    hx_attend_kernel<E, FP8, D, WR><<<(int)grid, AT_THREADS, lds, stream>>>(a);
    if (a.splits > 1) {
        const int64_t threads = (int64_t)a.n * a.kv.n_heads * a.max_q * a.group * (D / 4);
        hx_attend_join_kernel<E><<<(int)((threads + AT_THREADS - 1) / AT_THREADS), AT_THREADS, 0, stream>>>(a, C::ROWS);
    }
    return hx_check_launch(ctx, "hx_attend_kernel");
}

template <typename E, bool FP8, int D>
int plan(hx_ctx *ctx, AttendArgs &a, int max_len, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.max_q * a.group;
    const int wr = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
    const int tile_rows = 32 * wr, tile_keys = wr == 1 ? 128 : 64;
    a.row_tiles = (int)((rows + tile_rows - 1) / tile_rows);
    // few workgroups: the keys are divided too, two tiles at least to a part
    int64_t reach = max_len;
    if (a.window > 0 && reach > (int64_t)a.window + a.n_sink + a.max_q) reach = (int64_t)a.window + a.n_sink + a.max_q;
    const int64_t tiles = (reach + tile_keys - 1) / tile_keys, groups = (int64_t)a.n * a.kv.n_heads * a.row_tiles;
    int64_t splits = (2 * ctx->num_cu + groups - 1) / groups;
    if (splits > (tiles + 1) / 2) splits = (tiles + 1) / 2;
    if (splits > 64) splits = 64;
    a.splits = splits < 1 ? 1 : (int)splits;
    if (wr == 1) return launch<E, FP8, D, 1>(ctx, a, stream);
    if (wr == 2) return launch<E, FP8, D, 2>(ctx, a, stream);
    return launch<E, FP8, D, 4>(ctx, a, stream);
}

template <typename E, bool FP8>
int by_dim(hx_ctx *ctx, AttendArgs &a, int max_len, hipStream_t stream)
{
    if (a.kv.dim == 64) return plan<E, FP8, 64>(ctx, a, max_len, stream);
    if (a.kv.dim == 128) return plan<E, FP8, 128>(ctx, a, max_len, stream);
    return plan<E, FP8, 256>(ctx, a, max_len, stream);
}

template <typename E, bool FP8, int D, int WR>
int allow()
{
    using C = Tile<E, FP8, D, WR>;
    return hipFuncSetAttribute((const void *)hx_attend_kernel<E, FP8, D, WR>, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS + C::TREE) != hipSuccess;
}
template <typename E, bool FP8>
int allow_all()
{
    return allow<E, FP8, 64, 1>() | allow<E, FP8, 64, 2>() | allow<E, FP8, 64, 4>() | allow<E, FP8, 128, 1>() | allow<E, FP8, 128, 2>() |
           allow<E, FP8, 128, 4>() | allow<E, FP8, 256, 1>() | allow<E, FP8, 256, 2>() | allow<E, FP8, 256, 4>();
}

}  // namespace

// more LDS a workgroup than the 64 KB that need no asking
int hx_attend_init()
{
    return allow_all<__bf16, false>() | allow_all<__bf16, true>() | allow_all<_Float16, false>() | allow_all<_Float16, true>() ? HX_ERR_DEVICE : HX_OK;
}

extern "C" int hx_attend(hx_ctx *ctx, const hx_kv_pool *pool, int32_t layer, const hx_kv_seqs *seqs,
                         const hx_attend_args *args, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    KvView kv;
    if (int rc = hx_kv_view(ctx, pool, seqs, &kv)) return rc;
    HX_REQUIRE(ctx, args, HX_ERR_INVALID_ARG, "NULL arguments");
    const hx_attend_args &g = *args;
    HX_REQUIRE(ctx, layer >= 0 && layer < kv.n_layers, HX_ERR_INVALID_ARG, "layer %d of %d", layer, kv.n_layers);
    HX_REQUIRE(ctx, kv.dim == 64 || kv.dim == 128 || kv.dim == 256, HX_ERR_SHAPE, "head_dim %d is none of 64, 128, 256", kv.dim);
    HX_REQUIRE(ctx, g.n >= 0 && g.n_q >= 0 && g.max_q >= 0 && g.max_len >= 0 && g.window >= 0 && g.n_sink >= 0, HX_ERR_INVALID_ARG, "negative size");
    HX_REQUIRE(ctx, g.dtype == HX_BF16 || g.dtype == HX_F16, HX_ERR_INVALID_ARG, "queries of type %d", g.dtype);
    HX_REQUIRE(ctx, pool->dtype == HX_E4M3 || pool->dtype == g.dtype, HX_ERR_INVALID_ARG, "queries of type %d over a pool of type %d", g.dtype, pool->dtype);
    HX_REQUIRE(ctx, g.n_heads > 0 && g.n_heads % kv.n_heads == 0, HX_ERR_SHAPE, "%d query heads over %d KV heads", g.n_heads, kv.n_heads);
    HX_REQUIRE(ctx, !g.parent || g.max_q <= HX_MAX_DRAFTS, HX_ERR_SHAPE, "a tree of up to %d drafts, beyond %d", g.max_q, HX_MAX_DRAFTS);
    uint32_t scale_bits;                       // (this build's arithmetic tells no NaN)
    memcpy(&scale_bits, &g.scale, sizeof(scale_bits));
    HX_REQUIRE(ctx, (scale_bits & 0x7f800000u) != 0x7f800000u, HX_ERR_INVALID_ARG, "scale is not finite");
    if (g.n == 0 || g.n_q == 0 || g.max_q == 0) return HX_OK;
    HX_REQUIRE(ctx, g.q_ptr && g.q && g.out, HX_ERR_INVALID_ARG, "NULL array");
    HX_REQUIRE(ctx, (((uintptr_t)g.q | (uintptr_t)g.out) & 1) == 0, HX_ERR_INVALID_ARG, "q or out is not aligned to its type");
    HX_REQUIRE(ctx, kv.rows > 0, HX_ERR_INVALID_ARG, "%d sequences asked for of none", g.n);
    HX_REQUIRE(ctx, (int64_t)g.max_q * g.n_heads <= INT32_MAX / 2 && (int64_t)g.n * kv.n_heads <= INT32_MAX, HX_ERR_SHAPE,
               "%d queries of %d heads, %d sequences", g.max_q, g.n_heads, g.n);
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    hipStream_t stream = (hipStream_t)stream_;
    AttendArgs a{};
    a.kv = kv;
    a.layer = layer; a.n = g.n; a.row = g.row; a.q_ptr = g.q_ptr; a.n_q = g.n_q;
    a.max_q = g.max_q < g.n_q ? g.max_q : g.n_q;
    a.n_heads = g.n_heads; a.group = g.n_heads / kv.n_heads;
    a.q = g.q; a.q_token = g.q_token; a.q_head = g.q_head;
    a.out = g.out; a.out_token = g.out_token; a.out_head = g.out_head;
    a.lse = g.lse; a.scale = g.scale; a.window = g.window; a.n_sink = g.n_sink; a.parent = g.parent;
    a.k_scale = pool->k_scale; a.v_scale = pool->v_scale;
    a.q_wide = ((uintptr_t)g.q & 15) == 0 && g.q_token % 8 == 0 && g.q_head % 8 == 0;
    a.out_wide = ((uintptr_t)g.out & 7) == 0 && g.out_token % 4 == 0 && g.out_head % 4 == 0;
    const bool fp8 = pool->dtype == HX_E4M3;
    if (g.dtype == HX_BF16) return fp8 ? by_dim<__bf16, true>(ctx, a, g.max_len, stream) : by_dim<__bf16, false>(ctx, a, g.max_len, stream);
    return fp8 ? by_dim<_Float16, true>(ctx, a, g.max_len, stream) : by_dim<_Float16, false>(ctx, a, g.max_len, stream);
}
