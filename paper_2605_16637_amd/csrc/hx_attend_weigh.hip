// The weights that attention has given each cached token, summed over queries and heads.
#include "hx_attend_common.hpp"

namespace {

constexpr int WG_THREADS = 256, WG_WAVES = WG_THREADS / 64;
constexpr int BLOCKS = 2, KEYS = 16 * BLOCKS;                  // blocks of 16 keys, and keys, that a wavefront has at once

struct WeighArgs {
    AttendArgs a;
    float *weight;
    int64_t pitch;               // of a row's weights
    int each;                    // workgroups of a sequence
};

// Whether the row of entry i is listed before it too; all threads take part.
__device__ __forceinline__ bool row_before(const AttendArgs &a, int i)
{
    if (!a.row) return false;
    const int mine = a.row[i];
    bool hit = false;
    for (int k = threadIdx.x; k < i; k += WG_THREADS) hit |= a.row[k] == mine;
    return __syncthreads_or(hit);
}

// 8 numbers of a query, which need not be aligned to more than their type
template <typename E>
__device__ __forceinline__ typename Types<E>::x8 eight(const E *q)
{
    struct __attribute__((packed, aligned(2))) Loose { typename Types<E>::x8 x; };
    return ((const Loose *)q)->x;
}

// KEYS keys of a sequence from y0 on: where they lie, and those of them that are there.
struct Where {
    int64_t at[BLOCKS];
    uint32_t there;
};
template <int BITS, int D>
__device__ __forceinline__ Where where(const AttendArgs &a, const Seq &sq, const Extent &ex, int y0, int64_t page_bytes)
{
    using Pieces = KeyPieces<BITS, D>;
    const KvView &kv = a.kv;
    const int lane = threadIdx.x & 63, quad = lane >> 4, col = lane & 15, mine = y0 + (lane & (KEYS - 1));
    Where w;
    int page = -1;
    if (mine < ex.hi && (mine >= ex.lo || mine < a.n_sink)) page = sq.table[mine >> kv.shift];
    page = in_pool(kv, page);
    w.there = (uint32_t)__builtin_amdgcn_ballot_w64(page >= 0);
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        const int p = __shfl(page, b * 16 + col), y = y0 + b * 16 + col;
        // (what is not there reads the pool's first page, and counts for nothing)
        w.at[b] = (p < 0 ? 0 : p * page_bytes + (y & ((1 << kv.shift) - 1)) * ROW<BITS, D>) + quad * Pieces::BYTES;
    }
    return w;
}

// What a step needs: the keys of a head, and 16 rows (queries x query heads of the KV head) of it.
// A head's rows 16 at a time: with up to 16 query heads a KV head as many tokens as fit, with more a part of one token's.  A lane's row then has
// the same place in each, `at` behind the first: no division by the way.
struct RowTiles {
    int tokens, chunks, n;       // tokens of a row tile, or row tiles of a token; of a head
    __device__ __forceinline__ RowTiles(int nq, int group)
    {
        tokens = group < 16 ? 16 / group : 1;
        chunks = (group + 15) / 16;
        n = (nq + tokens - 1) / tokens * chunks;
    }
};
struct Place {
    static constexpr int NO_RANK = INT_MAX;
    int token, rank;             // of the row tile's; `rank` of those that may be missing, tokens or heads
    int64_t at;                  // in numbers of a layout
    __device__ __forceinline__ Place(int r, int group, const RowTiles &tiles, int64_t token_step, int64_t head_step)
    {
        token = r / group;                                        // (0 with 16 and more heads)
        rank = group > 16 ? r : token < tiles.tokens ? token : NO_RANK;
        at = rank < NO_RANK ? token * token_step + (r - token * group) * head_step : 0;
    }
};

template <int BITS, int D>
struct KeysOf {
    typename KeyPieces<BITS, D>::Piece k[BLOCKS][KeyPieces<BITS, D>::LOADS];
    uint32_t e[BLOCKS][KeyPieces<BITS, D>::LOADS];
};
template <typename E, int D>
struct RowsOf {
    typename Types<E>::x8 q[D / 32];
    float lse, unit;                 // unit: of the head's keys, of 8 bits
};

// 16 rows on their way to LDS, where each lane finds the pieces of its row.  They are asked for as rows lie in memory: a matrix operand's lanes beside
// each other hold different rows, of which each load by itself is an access of its own.
template <int D>
struct RowsInLds {
    static constexpr int CH = D / 8, LOADS = CH / 4, BYTES = 16 * CH * 16 + 256, RING = 3;
    static __device__ __forceinline__ int piece(int r, int c) { return r * CH + (c ^ (r & (CH < 16 ? CH - 1 : 15))); }
};

template <typename E, int BITS, int D>
struct Weigher {
    using Pieces = KeyPieces<BITS, D>;
    const AttendArgs &a;
    const Seq &sq;
    const char *k_at;
    const uint8_t *ke_at;
    int64_t head_bytes;
    int rows;                        // of a KV head
    const int *s_depth;
    const uint32_t *s_anc;
    float sum[BLOCKS][4];

    // (without `in` the same number of loads, of one place)
    __device__ __forceinline__ void ask_keys(KeysOf<BITS, D> &r, const Where &w, int head, bool in) const
    {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const int64_t at = in ? w.at[b] + head * head_bytes : 0;
#pragma unroll
            for (int l = 0; l < Pieces::LOADS; ++l) {
                r.k[b][l] = *(const typename Pieces::Piece *)(k_at + at + l * 64);
                r.e[b][l] = BITS == 4 ? ke_at[(at + l * 64) / 16] : 0;
            }
        }
    }
    // (few rows: all of a head; what is no row reads the first)
    __device__ __forceinline__ void ask_rows(RowsOf<E, D> &r, int head, int64_t q_at, int64_t lse_at) const
    {
        const int quad = threadIdx.x >> 4 & 3;
        const E *q = (const E *)a.q + (int64_t)sq.q0 * a.q_token + (int64_t)head * a.group * a.q_head + q_at;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) r.q[s] = eight(q + Pieces::place(s, quad));
        r.lse = a.lse[(int64_t)sq.q0 * a.n_heads + (int64_t)head * a.group + lse_at];
        r.unit = unit_of(head);
    }
    __device__ __forceinline__ float unit_of(int head) const
    {
        if constexpr (BITS != 8) return 1.0f;
        const float unit = (a.k_scale ? a.k_scale + a.layer * a.kv.n_heads : (const float *)a.zeros)[a.k_scale ? head : 0];
        return a.k_scale ? unit : 1.0f;
    }
    struct Operands {
        typedef uint32_t Words __attribute__((ext_vector_type(4)));
        Words x[BLOCKS][D / 32];
    };
    __device__ __forceinline__ void operands(Operands &o, const KeysOf<BITS, D> &k) const
    {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int l = 0; l < Pieces::LOADS; ++l)
#pragma unroll
                for (int j = 0; j < Pieces::EACH; ++j)
                    o.x[b][Pieces::EACH * l + j] = __builtin_bit_cast(typename Operands::Words, Pieces::template operand<E>(k.k[b][l], k.e[b][l], j));
    }
    // scores of the keys (a lane: keys 16 b + 4 quad + i) with the rows (its column)
    __device__ __forceinline__ void scores(const Operands &k, const RowsOf<E, D> &r, f32x4 (&s)[BLOCKS]) const
    {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            s[b] = f32x4{};
#pragma unroll
            for (int x = 0; x < D / 32; ++x) s[b] = mfma16(__builtin_bit_cast(typename Types<E>::x8, k.x[b][x]), r.q[x], s[b]);
        }
    }
    // t: this lane's row's token, counts: whether there is such a row; t_first, t_last: those of all lanes
    __device__ __forceinline__ void add(const f32x4 (&s)[BLOCKS], float lse, float unit, int t, bool counts, int t_first, int t_last, int y0, uint32_t there)
    {
        const int quad = threadIdx.x >> 4 & 3, end = y0 + KEYS - 1;
        const bool tree = a.parent != nullptr;
        const float sc = a.scale * unit;
        // as in attention the factor is no 0: a score of -infinity stays one
        const float c = copysignf(fmaxf(fabsf(sc), 1e-37f), sc) * LOG2E, less = -lse * LOG2E;
        const int first = tree ? sq.base - 1 : sq.base + t_first, last = tree ? sq.len : sq.base + t_last;
        counts = counts && __builtin_fabsf(lse) < __builtin_inff();
        if (there == 0xffffffffu && end <= first && (a.window <= 0 || end < a.n_sink || last - y0 < a.window)) {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[b][x], c, less));
                    sum[b][x] += counts ? p : 0.0f;
                }
        } else {
            const Sight view = sight(a, sq, t, s_depth, s_anc);
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int k = b * 16 + quad * 4 + x;
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[b][x], c, less));
                    sum[b][x] += counts && ((there >> k) & 1) && view.sees(y0 + k) ? p : 0.0f;
                }
        }
    }
    // over the 16 lanes that have a key's sums
    __device__ __forceinline__ void add_up()
    {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int d = 8; d > 0; d >>= 1) sum[b][x] += __shfl_xor(sum[b][x], d);
    }
};

// weight[row][y] += sum over the queries and heads that see key y of exp(score - lse): a query's softmax statistics are known, so a key's
// weight needs no other key's, no maximum and no second pass, and only keys are read.  One wavefront has a key's sums in a fixed order, and a
// sequence's row is another's to none: no atomics, the same sums every time.
//
// FEW: up to 16 rows a KV head, bound by the keys' bytes.  A wavefront takes 32 keys and all heads, so that its sums need no other's; two
// heads' keys are under way.  100 sequences over some 4000 tokens, 8 KV heads of 128: 264 us, 3.9 TB/s of keys (with the workgroup's wavefronts on
// a head each and their sums joined in LDS 303; at three wavefronts a SIMD 328, as the keys under way do not fit their registers).
// Else the wavefronts have the same 32 keys and divide heads and rows, 16 rows a step, and their sums are added in LDS: there are rows for many
// steps, and as few keys as possible a workgroup fill the chip.  Rows come through LDS, two steps ahead, and a head's keys are made operands
// once.  It mostly waits: for a head's first keys nothing else is under way.  The last 32 queries of 7
// prompts of some 6000 tokens, 32 heads of 128: 58 us, of which 9.5e6 vector instructions are some 15 of the chip's issue (their exponentials 4) and the
// matrix instructions 4; some 1290 workgroups have work, 1.7 rounds of three a CU.  That is at three wavefronts a SIMD, 67 at two; 75 with rows straight to registers, of which a load is an
// access for each of 64 lanes and every step waited for all loads; 95 with 128 keys a workgroup.
// a head and one of its row tiles
struct Step {
    int head, t0, chunk;
    __device__ __forceinline__ Step(int u, const RowTiles &tiles) : head(u / tiles.n), t0(u % tiles.n / tiles.chunks * tiles.tokens), chunk(u % tiles.chunks) {}
    __device__ __forceinline__ bool first() const { return (t0 | chunk) == 0; }
    // rows, or heads, that are left from here on
    __device__ __forceinline__ int left(int nq, int group) const { return group > 16 ? group - chunk * 16 : nq - t0; }
    // (behind the last one the first of the last head again)
    __device__ __forceinline__ void next(const RowTiles &tiles, int nq, int heads)
    {
        if (++chunk < tiles.chunks) return;
        chunk = 0;
        t0 += tiles.tokens;
        if (t0 < nq) return;
        t0 = 0;
        head += head + 1 < heads;
    }
};

template <typename E, int BITS, int D, bool FEW>
__global__ __launch_bounds__(WG_THREADS, D == 256 ? 1 : FEW ? 2 : 3) void hx_weigh_kernel(WeighArgs w)
{
    constexpr int TILE = FEW ? KEYS * WG_WAVES : KEYS;
    using Self = Weigher<E, BITS, D>;
    extern __shared__ __align__(16) char smem[];
    __shared__ __align__(16) char s_rows[FEW ? 1 : WG_WAVES][RowsInLds<D>::RING][FEW ? 16 : RowsInLds<D>::BYTES];
    int *s_depth = (int *)smem + HX_MAX_DRAFTS;
    uint32_t *s_anc = (uint32_t *)(s_depth + HX_MAX_DRAFTS);
    const AttendArgs &a = w.a;
    const KvView &kv = a.kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), quad = lane >> 4, col = lane & 15;
    const int i = blockIdx.x % a.n, part = blockIdx.x / a.n, H = kv.n_heads;
    Seq sq = sequence(a, i * H);
    sq.q0 = __builtin_amdgcn_readfirstlane(sq.q0);
    sq.nq = __builtin_amdgcn_readfirstlane(sq.nq);
    sq.len = __builtin_amdgcn_readfirstlane(sq.len);
    sq.base = __builtin_amdgcn_readfirstlane(sq.base);
    const Extent ex = extent<TILE>(a, sq, 0, sq.nq - 1);
    if (!sq.ok) { if (tid == 0 && part == 0 && (!sq.there || sq.nq > 0)) hx_raise(kv.status, HX_ERR_INDEX); return; }
    if (sq.nq == 0 || part >= ex.n) return;
    if (row_before(a, i)) { if (tid == 0 && part == 0) hx_raise(kv.status, HX_ERR_INDEX); return; }
    if (a.parent) plant(a, sq, (int *)smem, s_depth, s_anc);
    const int64_t page_bytes = ((int64_t)H << kv.shift) * ROW<BITS, D>, here = (int64_t)a.layer * kv.n_pages * page_bytes;
    Self g{a, sq, (const char *)kv.k + here, BITS == 4 ? a.k_exp + here / 16 : nullptr, (int64_t)ROW<BITS, D> << kv.shift, sq.nq * a.group, s_depth, s_anc, {}};
    float *to = w.weight + (a.row ? a.row[i] : i) * w.pitch;
    // where the rows of a row tile lie that this lane asks for, in bytes, if they may be read 16 bytes at a time and are not far apart
    const RowTiles tiles(sq.nq, a.group);
    const Place mine(col, a.group, tiles, a.n_heads, 1);
    const bool wide = a.q_wide && a.q_token >= 0 && a.q_head >= 0 && a.q_token < 1 << 24 && a.q_head < 1 << 24;
    int near[RowsInLds<D>::LOADS], far[RowsInLds<D>::LOADS], rank[RowsInLds<D>::LOADS];
#pragma unroll
    for (int j = 0; j < RowsInLds<D>::LOADS; ++j) {
        const int r = (j * 64 + lane) / RowsInLds<D>::CH;
        const Place p(r, a.group, tiles, a.q_token, a.q_head);
        near[j] = (RowsInLds<D>::piece(r, lane % RowsInLds<D>::CH) - r * RowsInLds<D>::CH) * 16;
        far[j] = (int)p.at * 2;
        rank[j] = p.rank;
    }
    for (int tile = part; tile < ex.n; tile += w.each) {
        const int y0 = (tile < ex.sink_tiles ? tile : tile - ex.sink_tiles + ex.lo_tile) * TILE + (FEW ? wave * KEYS : 0);
        const Where at = where<BITS, D>(a, sq, ex, y0, page_bytes);
        if (at.there == 0) continue;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int x = 0; x < 4; ++x) g.sum[b][x] = 0.0f;
        if constexpr (FEW) {
            KeysOf<BITS, D> k0, k1;
            RowsOf<E, D> r0, r1;
            g.ask_keys(k0, at, 0, true);
            const int t = col / a.group;
            const bool is_row = col < g.rows;
            const int64_t q_at = is_row ? t * a.q_token + (col - t * a.group) * a.q_head : 0, lse_at = is_row ? (int64_t)t * a.n_heads + (col - t * a.group) : 0;
            g.ask_rows(r0, 0, q_at, lse_at);
            g.ask_keys(k1, at, 1, H > 1);
            g.ask_rows(r1, H > 1 ? 1 : 0, q_at, lse_at);
            auto step = [&](KeysOf<BITS, D> &k, RowsOf<E, D> &r, int head) {
                f32x4 s[BLOCKS];
                typename Self::Operands now;
                g.operands(now, k);
                g.scores(now, r, s);
                const float lse = r.lse, unit = r.unit;
                g.ask_keys(k, at, head + 2, head + 2 < H);
                g.ask_rows(r, head + 2 < H ? head + 2 : head, q_at, lse_at);
                g.add(s, lse, unit, t, is_row, 0, sq.nq - 1, y0, at.there);
            };
            // (a step that may be left out would have all loads waited for)
            int head = 0;
            for (; head + 1 < H; head += 2) {
                step(k0, r0, head);
                step(k1, r1, head + 1);
            }
            if (head < H) step(k0, r0, head);
            g.add_up();
        } else {
            using Q = RowsInLds<D>;
            const int steps = H * tiles.n, u0 = (int)((int64_t)steps * wave / WG_WAVES), u1 = (int)((int64_t)steps * (wave + 1) / WG_WAVES);
            if (u0 < u1) {
                Step to(u0, tiles), from = to;
                int put = 0, get = 0;
                auto ask = [&] {
                    char *slot = s_rows[wave][put];
                    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(slot));
                    const int left = to.left(sq.nq, a.group);
                    const int64_t token = sq.q0 + to.t0, qhead = to.head * a.group + to.chunk * 16;
                    const E *q = (const E *)a.q + token * a.q_token + qhead * a.q_head;
                    if (wide)
#pragma unroll
                        for (int j = 0; j < Q::LOADS; ++j) to_lds(lds + j * 1024, near[j] + (rank[j] < left ? far[j] : 0), (const char *)q);
                    else
                        for (int j = 0; j < Q::LOADS; ++j) {
                            const int r = (j * 64 + lane) / Q::CH, c = Q::piece(r, lane % Q::CH) - r * Q::CH;
                            const Place p(r, a.group, tiles, a.q_token, a.q_head);
                            *(typename Types<E>::x8 *)(slot + j * 1024 + lane * 16) = eight(q + (p.rank < left ? p.at : 0) + c * 8);
                        }
                    to_lds_word(lds + Q::LOADS * 1024, mine.rank < left ? (int)mine.at * 4 : 0, (const char *)(a.lse + token * a.n_heads + qhead));
                    put = put + 1 < Q::RING ? put + 1 : 0;
                    to.next(tiles, sq.nq, H);              // (always as many loads are under way)
                };
#pragma unroll
                for (int x = 0; x < Q::RING - 1; ++x) ask();
                for (int u = u0; u < u1;) {
                    float unit = g.unit_of(from.head);
                    typename Self::Operands k;
                    {
                        KeysOf<BITS, D> stored;
                        g.ask_keys(stored, at, from.head, true);
                        g.operands(k, stored);
                    }
                    // (waited for here, or the compiler would at every step, and for the rows under way)
                    asm volatile("" : "+v"(unit));
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                        for (int x = 0; x < D / 32; ++x) asm volatile("" : "+v"(k.x[b][x]));
#pragma unroll 1
                    do {
                        // these rows are there, and what was read where the next will be has come
                        if (wide) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((Q::RING - 2) * (Q::LOADS + 1)) : "memory");
                        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                        ask();
                        const char *slot = s_rows[wave][get];
                        RowsOf<E, D> r;
#pragma unroll
                        for (int s = 0; s < D / 32; ++s) r.q[s] = *(const typename Types<E>::x8 *)(slot + Q::piece(col, KeyPieces<BITS, D>::place(s, quad) / 8) * 16);
                        r.lse = *(const float *)(slot + Q::LOADS * 1024 + col * 4);
                        f32x4 s[BLOCKS];
                        g.scores(k, r, s);
                        const int t_last = from.t0 + tiles.tokens < sq.nq ? from.t0 + tiles.tokens - 1 : sq.nq - 1;
                        g.add(s, r.lse, unit, from.t0 + mine.token, mine.rank < from.left(sq.nq, a.group), from.t0, t_last, y0, at.there);
                        get = get + 1 < Q::RING ? get + 1 : 0;
                        from.next(tiles, sq.nq, H);
                    } while (++u < u1 && !from.first());
                }
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            }
            g.add_up();
            __shared__ float s_sum[WG_WAVES][KEYS];
            if (col == 0)
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int x = 0; x < 4; ++x) s_sum[wave][b * 16 + quad * 4 + x] = g.sum[b][x];
            __syncthreads();
            if (tid < KEYS && ((at.there >> tid) & 1)) {
                float all = s_sum[0][tid];
#pragma unroll
                for (int v = 1; v < WG_WAVES; ++v) all += s_sum[v][tid];
                to[y0 + tid] += all;
            }
            __syncthreads();
            continue;
        }
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const int k = b * 16 + quad * 4 + col;
            const float (&sum)[4] = g.sum[b];
            if (col < 4 && ((at.there >> k) & 1)) to[y0 + k] += col == 0 ? sum[0] : col == 1 ? sum[1] : col == 2 ? sum[2] : sum[3];
        }
    }
}

template <typename E, int BITS, int D, bool FEW>
int launch(hx_ctx *ctx, WeighArgs &w, int max_len, hipStream_t stream)
{
    const int tile = FEW ? KEYS * WG_WAVES : KEYS;
    int64_t reach = max_len;
    const HxAttend &a = w.a;
    if (a.window > 0 && reach > (int64_t)a.window + a.n_sink + a.max_q) reach = (int64_t)a.window + a.n_sink + a.max_q;
    const int64_t tiles = (reach + tile - 1) / tile + 2, most = hx_most_groups(WG_THREADS) / a.n;
    w.each = (int)(tiles < most ? tiles : most);
    const int lds = a.parent ? HX_MAX_DRAFTS * 4 + TREE_BYTES : 0;
    hx_weigh_kernel<E, BITS, D, FEW><<<(int)((int64_t)w.each * a.n), WG_THREADS, lds, stream>>>(w);
    return hx_check_launch(ctx, "hx_weigh_kernel");
}

template <typename E, int BITS, int D>
int by_rows(hx_ctx *ctx, WeighArgs &w, int max_len, hipStream_t stream)
{
    return (int64_t)w.a.max_q * w.a.group <= 16 ? launch<E, BITS, D, true>(ctx, w, max_len, stream) : launch<E, BITS, D, false>(ctx, w, max_len, stream);
}

template <typename E, int BITS>
int by_dim(hx_ctx *ctx, WeighArgs &w, int max_len, hipStream_t stream)
{
    if (w.a.kv.dim == 64) return by_rows<E, BITS, 64>(ctx, w, max_len, stream);
    if (w.a.kv.dim == 128) return by_rows<E, BITS, 128>(ctx, w, max_len, stream);
    return by_rows<E, BITS, 256>(ctx, w, max_len, stream);
}

template <typename E>
int by_type(hx_ctx *ctx, int pool_dtype, WeighArgs &w, int max_len, hipStream_t stream)
{
    if (pool_dtype == HX_E4M3) return by_dim<E, 8>(ctx, w, max_len, stream);
    if (pool_dtype == HX_E2M1) return by_dim<E, 4>(ctx, w, max_len, stream);
    return by_dim<E, 16>(ctx, w, max_len, stream);
}

}  // namespace

extern "C" int hx_kv_weigh(hx_ctx *ctx, const hx_kv_pool *pool, int32_t layer, const hx_kv_seqs *seqs,
                           const hx_attend_args *args, float *weight, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    KvView kv;
    bool any;
    if (int rc = hx_kv_view(ctx, pool, seqs, &kv)) return rc;
    if (int rc = hx_attend_check(ctx, pool, layer, kv, args, false, &any)) return rc;
    if (!any) return HX_OK;
    HX_REQUIRE(ctx, args->lse && weight, HX_ERR_INVALID_ARG, "NULL lse or weights");
    HX_REQUIRE(ctx, (((uintptr_t)args->lse | (uintptr_t)weight) & 3) == 0, HX_ERR_INVALID_ARG, "lse or weights are not aligned to their type");
    HX_REQUIRE(ctx, args->n <= hx_most_groups(WG_THREADS), HX_ERR_SHAPE, "%d sequences in one call", args->n);
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    WeighArgs w{hx_attend_view(ctx, pool, layer, kv, *args), weight, (int64_t)kv.max_pages << kv.shift, 1};
    return args->dtype == HX_BF16 ? by_type<__bf16>(ctx, pool->dtype, w, args->max_len, (hipStream_t)stream_)
                                  : by_type<_Float16>(ctx, pool->dtype, w, args->max_len, (hipStream_t)stream_);
}
