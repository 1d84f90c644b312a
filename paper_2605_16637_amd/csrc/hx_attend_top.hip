// Attention over the pages that every query chooses for every KV head: what a page's keys can score at most, the pages of the largest of these,
// and hx_attend's kernels over them, for which each query and KV head is a sequence with a table of its own.
#include "hx_attend_common.hpp"
#include "hx_nth.hpp"

namespace {

constexpr int TOP_THREADS = 256, TOP_WAVES = TOP_THREADS / 64;
constexpr int64_t TOP_ROOM = (int64_t)1 << 28;           // bytes of scores and of chosen pages at once

struct TopArgs {
    AttendArgs a;
    const void *bounds;              // of the layer
    int first_query, n_queries;      // of this part of the call
    int n_pages, n_first, n_last;
    int picked_pages;                // n_pages, or a row's entries where they are fewer
    int stride;                      // entries of a row, up to a multiple of 16; 0 where no row has more than n_pages entries
    float *score;                    // [query][KV head][stride]
    float *off;                      // [query][KV head][stride / 16] what a score of these 16 pages may be off by
    double *exact;                   // [query][KV head][stride] of those pages for which that matters
    int32_t *picked, *picked_len;    // what hx_attend's kernels read
    int32_t *chosen;                 // of the call's first query, or NULL
    int q_tiles, chunks;             // of a sequence; workgroups that look at the pages of a tile of queries and a KV head
};

// A query's row: its pages up to its own, `own`.
struct Place {
    bool ok, none;                   // none: no sequence has such a query
    int pos, own;
    const int32_t *table;
};
__device__ __forceinline__ Place place(const AttendArgs &a, int j)
{
    int lo = 0, hi = a.n - 1;
    // with one query a sequence it is the j-th
    const int guess = j < hi ? j : hi;
    if (a.q_ptr[guess] <= j && a.q_ptr[guess + 1] > j) lo = hi = guess;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.q_ptr[mid] <= j) lo = mid; else hi = mid - 1;
    }
    const Seq s = sequence(a, lo * a.kv.n_heads);
    Place p;
    p.ok = s.ok && j >= s.q0 && j < s.q0 + s.nq;
    p.none = j < a.q_ptr[0] || j >= a.q_ptr[a.n];
    p.pos = p.ok ? s.base + j - s.q0 : 0;
    p.own = p.pos >> a.kv.shift;
    p.table = s.table;
    return p;
}

// ---- what a page can score ---------------------------------------------------

constexpr float INF = __builtin_inff();
typedef short s16x8 __attribute__((ext_vector_type(8)));

// bounds as numbers of the queries' type; those of 8 and 4 bits are bf16, and fp16 exactly
template <typename Q, typename E>
__device__ __forceinline__ typename Types<Q>::x8 as_query(typename Types<E>::x8 x)
{
    if constexpr (std::is_same_v<Q, E>) return x;
    else {
        typename Types<Q>::x8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (Q)(float)x[i];
        return y;
    }
}

// What pages can score, by the matrix units: a query's numbers that are not below 0 times the upper bounds, and the others times the lower ones.  Products
// of 16-bit numbers are exact and their sums are held in 32 bits, so a score is off by at most 2 D 2^-23 of the sum of its terms' sizes, which |q|
// times the larger bound's size sums to: where that could change which pages are chosen, they are scored again in 64 bits.
//
// ONE: a single query a sequence, whose heads are the columns; else 16 queries beside each other are, and the heads follow each other.  A wavefront has 16
// pages at once and asks for the next 16.  Bound by the bounds' bytes with one query a sequence: 48 of them over some 16000 tokens, pages of 32, 8 heads of
// 128: 126 MB in 39 us, 3.2 TB/s; 602 queries over some 8000: 16 us.  With all scores in 64 bits by the vector units the whole calls took 240 and 384 us where
// they took 157 and 157 with these.
template <typename Q, typename E, int D, bool ONE>
__global__ __launch_bounds__(TOP_THREADS) void hx_top_score_kernel(TopArgs t)
{
    using Q8 = typename Types<Q>::x8;
    using E8 = typename Types<E>::x8;
    constexpr int PARTS = D / 32;
    const AttendArgs &a = t.a;
    const KvView &kv = a.kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quad = lane >> 4, col = lane & 15;
    const int pairs = a.n * kv.n_heads, pair = blockIdx.x % pairs, rest = blockIdx.x / pairs, head = pair % kv.n_heads;
    const int qt = rest % t.q_tiles, part = rest / t.q_tiles;
    const Seq sq = sequence(a, pair);
    if (!sq.ok) return;
    // the tile's queries that are of this part of the call
    int t0 = ONE ? qt : qt * 16, t1 = ONE ? qt + 1 : qt * 16 + 16;
    t1 = t1 < sq.nq ? t1 : sq.nq;
    const int from = t.first_query - sq.q0, until = from + t.n_queries;
    if (t0 >= t1 || t1 <= from || t0 >= until) return;
    const int last_seen = t1 <= until ? t1 - 1 : until - 1, own = (sq.base + last_seen) >> kv.shift, last = own - t.n_last;
    if (own < t.n_pages) return;                                  // (no more pages than they may see)
    const int mine = ONE ? t0 : t0 + col;                         // this column's query
    const bool real = mine >= from && mine < until && mine < sq.nq;
    const int64_t line = real ? (int64_t)(mine - from) * kv.n_heads + head : 0;
    const int rounds = ONE ? (a.group + 15) / 16 : a.group;
    constexpr float UNIT = 2.0f * D * 1.1920929e-07f * 1.02f;

    const int steps = (last + 16) / 16 - t.n_first / 16;          // 16 pages each, from the one with the first that is not seen in any case
    const int stride = t.chunks * TOP_WAVES;
    auto look = [&](int step) {
        const int b = (t.n_first / 16 + step) * 16 + col;
        return step < steps && b <= last && b >= t.n_first ? sq.table[b] : -1;
    };
    E8 lo[PARTS], hi[PARTS];
    unsigned here = 0;                                            // which of the 16 pages are there
    auto fetch = [&](int page) {
        page = in_pool(kv, page);
        here = (unsigned)__builtin_amdgcn_ballot_w64(page >= 0) & 0xffffu;
        const E *at = (const E *)t.bounds + ((int64_t)(page < 0 ? 0 : page) * kv.n_heads + head) * (2 * D) + quad * 8;
#pragma unroll
        for (int s = 0; s < PARTS; ++s) { lo[s] = *(const E8 *)(at + s * 32); hi[s] = *(const E8 *)(at + D + s * 32); }
    };
    int step = part * TOP_WAVES + wave;
    if (step >= steps) return;
    int next = look(step + stride);
    fetch(look(step));
    for (; step < steps; step += stride) {
        const unsigned now = here;
        Q8 l[PARTS], h[PARTS];
        s16x8 m[PARTS];
#pragma unroll
        for (int s = 0; s < PARTS; ++s) {
            l[s] = as_query<Q, E>(lo[s]);
            h[s] = as_query<Q, E>(hi[s]);
            const s16x8 x = __builtin_bit_cast(s16x8, l[s]) & (short)0x7fff, y = __builtin_bit_cast(s16x8, h[s]) & (short)0x7fff;
            m[s] = __builtin_elementwise_max(x, y);
        }
        if (step + stride < steps) {
            fetch(next);
            next = look(step + 2 * stride);
        }
        float best[4] = {-INF, -INF, -INF, -INF}, off = 0.0f;
        for (int r = 0; r < rounds; ++r) {
            const int g = ONE ? r * 16 + col : r;
            const bool in = real && g < a.group;
            const Q *q = (const Q *)a.q + (int64_t)(sq.q0 + (in ? mine : t0)) * a.q_token + (int64_t)(head * a.group + (in ? g : 0)) * a.q_head + quad * 8;
            f32x4 acc = {}, size = {};
#pragma unroll
            for (int s = 0; s < PARTS; ++s) {
                Q8 x = {};
                if (in) {
                    if (a.q_wide) x = *(const Q8 *)(q + s * 32);
                    else
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = q[s * 32 + i];
                }
                s16x8 bits = __builtin_bit_cast(s16x8, x);
                if (a.scale < 0) bits ^= (short)0x8000;
                const s16x8 under = bits >> 15;                   // all bits set where it is below 0 (or -0, times anything)
                acc = mfma16(h[s], __builtin_bit_cast(Q8, (s16x8)(bits & ~under)), acc);
                acc = mfma16(l[s], __builtin_bit_cast(Q8, (s16x8)(bits & under)), acc);
                size = mfma16(__builtin_bit_cast(Q8, m[s]), __builtin_bit_cast(Q8, (s16x8)(bits & (short)0x7fff)), size);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!in || !((now >> (quad * 4 + i)) & 1)) continue;
                best[i] = fmaxf(best[i], acc[i]);
                // (an infinity or NaN in a score makes it worth nothing)
                const float by = __builtin_fabsf(acc[i]) < INF ? size[i] : INF;
                off = by < off ? off : by == by ? by : INF;
            }
        }
        if constexpr (ONE)
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) best[i] = fmaxf(best[i], __shfl_xor(best[i], d));
                off = fmaxf(off, __shfl_xor(off, d));
            }
        off = fmaxf(off, lane_16_away(off));
        off = fmaxf(off, other_half(off));
        const int block = t.n_first / 16 + step;
        if (real && (!ONE || col == 0)) {
            *(float4 *)(t.score + line * t.stride + block * 16 + quad * 4) = make_float4(best[0], best[1], best[2], best[3]);
            if (quad == 0) t.off[line * (t.stride / 16) + block] = off * UNIT + 1e-37f;
        }
    }
}

// ---- the pages of the largest ------------------------------------------------

__device__ __forceinline__ double across(double x, int d)
{
    const uint64_t v = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __shfl_xor((uint32_t)v, d), hi = __shfl_xor((uint32_t)(v >> 32), d);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// A page's score in 64 bits by D / 8 lanes beside each other, of which each has 8 places: the same products, whose sums are off by some 2^-50 of their terms.
template <typename Q, typename E, int D>
__device__ __forceinline__ double exact_score(const TopArgs &t, int j, int head, int page, int sub)
{
    using Q8 = typename Types<Q>::x8;
    using E8 = typename Types<E>::x8;
    const AttendArgs &a = t.a;
    const E *at = (const E *)t.bounds + ((int64_t)page * a.kv.n_heads + head) * (2 * D) + sub * 8;
    const E8 lo = *(const E8 *)at, hi = *(const E8 *)(at + D);
    double best = -__builtin_inf();
#pragma unroll 1
    for (int g0 = 0; g0 < a.group; g0 += 4) {
        Q8 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const Q *q = (const Q *)a.q + (int64_t)j * a.q_token + (int64_t)(head * a.group + (g0 + k < a.group ? g0 + k : g0)) * a.q_head + sub * 8;
            if (a.q_wide) x[k] = *(const Q8 *)q;
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) x[k][i] = q[i];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            double v = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = a.scale < 0 ? -(float)x[k][i] : (float)x[k][i];
                v = fma((double)y, (double)(float)(y < 0 ? lo[i] : hi[i]), v);
            }
#pragma unroll
            for (int d = D / 16; d > 0; d >>= 1) v += across(v, d);
            best = fmax(best, v == v ? v : __builtin_inf());      // a bound that is no number is taken for +infinity
        }
    }
    return best;
}

// Keys of scores, 0 where they are -infinity (-0 and 0 are the same number).
__device__ __forceinline__ uint64_t key_of(double x) { return x == -__builtin_inf() ? 0 : nth_key(x + 0.0); }
__device__ __forceinline__ uint32_t key_of(float x)
{
    const int32_t v = __builtin_bit_cast(int32_t, x + 0.0f);
    return x == -INF ? 0 : (uint32_t)(v ^ (v >> 31 | INT32_MIN));
}
__device__ __forceinline__ float of_key(uint32_t k)
{
    const int32_t v = (int32_t)k;
    return __builtin_bit_cast(float, v < 0 ? v ^ INT32_MIN : ~v);
}

// A workgroup a query and KV head, of up to 256 pages a single wavefront, which needs no barriers: a chain of round trips (the query's row, its length, its
// pages and their scores, all of which are kept in LDS) and of passes over the scores.  cache: pages that fit there.  One query over 30000 tokens, 64 pages of
// 1875 for each of 8 heads: 17 us, of which the row and its scores take 5, the limit 4 and the scores in 64 bits 5; 384 such of 512: 19.5.  (The limit found
// by quarters, at half the meetings but three times the counts, takes as long.)
template <typename Q, typename E, int D, int THREADS>
__global__ __launch_bounds__(THREADS) void hx_top_pick_kernel(TopArgs t, int cache)
{
    constexpr int WAVES = THREADS / 64, LANES = D / 8, LIST = 64, EACH = 4;      // EACH: scores that a thread holds
    __shared__ NthHeld<uint32_t, THREADS> s_near;
    __shared__ NthHeld<uint64_t, THREADS> s_far;
    __shared__ NthState<uint64_t, THREADS> s_many;
    __shared__ uint64_t s_key[LIST];
    __shared__ int s_list[LIST], s_n_list, s_count[2][WAVES];
    __shared__ float s_off[WAVES];
    extern __shared__ int s_pages[];                               // [cache] entries of the row, then their scores
    float *s_score = (float *)(s_pages + cache);
    const AttendArgs &a = t.a;
    const KvView &kv = a.kv;
    const int pair = blockIdx.x, head = pair % kv.n_heads, j = t.first_query + pair / kv.n_heads;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Place p = place(a, j);
    int32_t *picked = t.picked + (int64_t)pair * t.picked_pages;
    int32_t *chosen = t.chosen ? t.chosen + ((int64_t)j * kv.n_heads + head) * t.n_pages : nullptr;
    if (p.none) {
        if (tid == 0) t.picked_len[pair] = -1;
        return;
    }
    if (!p.ok) {
        if (tid == 0) { hx_raise(kv.status, HX_ERR_INDEX); picked[0] = -1; t.picked_len[pair] = 1; }
        if (chosen)
            for (int i = tid; i < t.n_pages; i += THREADS) chosen[i] = -1;
        return;
    }
    // sums of x and y over the wavefronts, each of which has one
    auto add_up = [&](int &x, int &y) {
        if constexpr (WAVES > 1) {
            if (lane == 0) { s_count[0][wave] = x; s_count[1][wave] = y; }
            __syncthreads();
            x = y = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) { x += s_count[0][w]; y += s_count[1][w]; }
            __syncthreads();
        }
    };
    const HxSeen seen = hx_seen_in_any_case(p.own, t.n_pages, t.n_first, t.n_last);
    const bool all = seen.all || kv.n_pages == 0;
    const int from = seen.from, to = seen.to;                      // the pages between those that are seen in any case
    const float *score = t.score + (int64_t)pair * t.stride;
    double *exact = t.exact + (int64_t)pair * t.stride;
    const bool cached = p.own < cache;
    float off = 0.0f;
    if (!all)
        for (int i = from / 16 + tid; i <= (to - 1) / 16; i += THREADS) off = fmaxf(off, t.off[(int64_t)pair * (t.stride / 16) + i]);
    int fixed = 0, none = 0;                                       // pages that are there of those seen in any case
    if (cached) {
        for (int b0 = 0; b0 <= p.own; b0 += THREADS) {
            const int b = b0 + tid;
            const bool in = b <= p.own, between = !all && b >= from && b < to;
            const int page = in_pool(kv, in ? p.table[b] : -1);
            if (in) s_pages[b] = page;
            if (between) s_score[b] = score[b];
            fixed += __builtin_popcountll(__builtin_amdgcn_ballot_w64(!between && page >= 0));
        }
    } else if (!all)
        // (a row that all of is seen need not have as many entries)
        for (int i0 = 0; i0 < seen.fixed; i0 += THREADS) {
            const int i = i0 + tid, page = i < seen.fixed ? p.table[seen.entry(i)] : -1;
            fixed += __builtin_popcountll(__builtin_amdgcn_ballot_w64(page >= 0 && page < kv.n_pages));
        }
    add_up(fixed, none);
    auto score_of = [&](int b) { return cached ? s_score[b] : score[b]; };
    auto page_at = [&](int b) {
        if (cached) return s_pages[b];
        const int page = p.table[b];
        return page < kv.n_pages ? page : -1;
    };
    // which of the pages between are taken
    enum { NONE, LEFT, NEAR, MARKED, EXACT, BLIND } how = NONE;    // none; all that are there; scores from `under` on; scores above `over` and infinite
    float over = INF, under = INF;                                 // ones; above `over` and, from `under` on, the largest exact ones; all by their exact ones
    uint64_t edge = 0;
    int equals = 0, unsures = 0;
    // (a page that is not there has a score of -infinity, which `under` may be of numbers near the type's lowest)
    auto unsure = [&](int b) {
        if (how == BLIND) return page_at(b) >= 0;
        const float x = score_of(b);
        return x <= over && x >= under && x > -INF;
    };
    const int want = t.n_pages - fixed;
    if (!all && want > 0) {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) off = fmaxf(off, __shfl_xor(off, d));
        if (lane == 0) s_off[wave] = off;
        if (tid == 0) s_n_list = 0;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) off = fmaxf(off, s_off[w]);
        if (off < INF) {
            uint32_t k;
            if (to - from <= EACH * THREADS) {
                uint32_t x[EACH];
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const int b = from + i * THREADS + tid;
                    x[i] = b < to ? key_of(score_of(b)) : 0;
                }
                nth_largest_held(x, want, s_near, &k, &equals);
            } else {
                nth_largest([&](int b) { return (uint64_t)key_of(score_of(b)); }, from, to, want, s_many);
                k = (uint32_t)s_many.edge;
            }
            how = k ? EXACT : LEFT;
            const float near = of_key(k);
            over = near + 2.1f * off;
            under = near - 2.1f * off;
        } else how = BLIND;
        int sure = 0;
        if (how != LEFT) {
            for (int b0 = from; b0 < to; b0 += THREADS) {
                const int b = b0 + tid;
                const bool u = b < to && unsure(b);
                sure += __builtin_popcountll(__builtin_amdgcn_ballot_w64(b < to && how == EXACT && score_of(b) > over));
                unsures += __builtin_popcountll(__builtin_amdgcn_ballot_w64(u));
                if (u) {
                    const int at = atomicAdd(&s_n_list, 1);
                    if (at < LIST) s_list[at] = b;
                }
            }
            add_up(sure, unsures);
        }
        if (how == EXACT && sure + unsures == want) how = NEAR;
        if (how >= EXACT) {
            __syncthreads();
            const int groups = THREADS / LANES, sub = tid % LANES;
            if (unsures <= LIST) {
                for (int i0 = 0; i0 < unsures; i0 += groups) {
                    const int i = i0 + tid / LANES, b = s_list[i < unsures ? i : 0];
                    const double x = exact_score<Q, E, D>(t, j, head, page_at(b), sub);
                    if (i < unsures && sub == 0) s_key[i] = key_of(x);
                }
                __syncthreads();
                const uint64_t mine = tid < unsures ? s_key[tid] : 0;
                if (cached) {
                    // each counts those before it; scores say from here on whether their page is taken
                    if (tid < unsures) {
                        const int b = s_list[tid];
                        int before = 0;
                        for (int i = 0; i < unsures; ++i) before += s_key[i] > mine || (s_key[i] == mine && s_list[i] < b);
                        s_score[b] = mine > 0 && before < want - sure ? INF : -INF;
                    }
                    __syncthreads();
                    how = MARKED;
                } else {
                    const uint64_t x[1] = {mine};
                    nth_largest_held(x, want - sure, s_far, &edge, &equals);
                }
            } else {
                for (int b0 = from; b0 < to; b0 += groups) {
                    const int b = b0 + tid / LANES, page = b < to && unsure(b) ? page_at(b) : -1;
                    const double x = exact_score<Q, E, D>(t, j, head, page < 0 ? 0 : page, sub);
                    if (page >= 0 && sub == 0) exact[b] = x;
                }
                __syncthreads();
                nth_largest([&](int b) { return unsure(b) ? key_of(exact[b]) : (uint64_t)0; }, from, to, want - sure, s_many);
                edge = s_many.edge;
                equals = s_many.equals;
            }
        }
    }
    auto exact_key = [&](int b) {
        if (unsures > LIST) return key_of(exact[b]);
        int i = 0;
        while (i < unsures - 1 && s_list[i] != b) ++i;
        return s_key[i];
    };
    // the pages in rising order
    int n = 0, seen_equal = 0, turn = 0;
    for (int b0 = 0; b0 <= p.own; b0 += THREADS) {
        const int b = b0 + tid;
        const int page = cached ? (b <= p.own ? s_pages[b] : -1) : in_pool(kv, b <= p.own ? p.table[b] : -1);
        const bool between = !all && b >= from && b < to && page >= 0;
        const bool told = between && how >= EXACT && unsure(b);
        const float x = between && how != NONE ? score_of(b) : 0.0f;
        const uint64_t k = told ? exact_key(b) : 0;
        const bool equal = k == edge && k > 0;
        const bool best = told ? k > edge : how == LEFT ? x > -INF : how == NEAR ? x >= under : how == MARKED ? x > over || x == INF : how == EXACT && x > over;
        const bool sure = page >= 0 && (!between || best);
        // the wavefronts' counts, of which each adds up those before it: of equal ones the first are taken
        const unsigned long long e = __builtin_amdgcn_ballot_w64(equal);
        int all_sure = __builtin_popcountll(__builtin_amdgcn_ballot_w64(sure)), all_equal = __builtin_popcountll(e);
        int rank = seen_equal + __builtin_popcountll(e & ((1ull << lane) - 1)), at = n;
        auto of_equal = [&](int before, int here) { const int left = equals - before; return left < 0 ? 0 : left < here ? left : here; };
        if constexpr (WAVES > 1) {
            if (lane == 0) s_count[turn][wave] = all_sure << 16 | all_equal;
            __syncthreads();
            rank -= seen_equal;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const int c = s_count[turn][w], taken = (c >> 16) + of_equal(seen_equal, c & 0xffff);
                n += taken;
                at += w < wave ? taken : 0;
                rank += w == wave ? seen_equal : 0;
                seen_equal += c & 0xffff;
            }
            turn ^= 1;                                             // (who is still reading the other has passed a barrier since)
        } else {
            n += all_sure + of_equal(seen_equal, all_equal);
            seen_equal += all_equal;
        }
        const bool take = sure || (equal && rank < equals);
        at += __builtin_popcountll(__builtin_amdgcn_ballot_w64(take) & ((1ull << lane) - 1));
        if (take) {
            picked[at] = page;
            if (chosen) chosen[at] = b;
            // where its own page is there it is the last of all; else all that are chosen are full
            if (b == p.own) t.picked_len[pair] = (at << kv.shift) + (p.pos & ((1 << kv.shift) - 1)) + 1;
        }
        if (b == p.own && !take) {
            if (at == 0) picked[0] = -1;
            t.picked_len[pair] = at == 0 ? 1 : at << kv.shift;
        }
    }
    if (chosen)
        for (int i = n + tid; i < t.n_pages; i += THREADS) chosen[i] = -1;
}

template <typename Q, typename E, int D>
void score_and_pick(const TopArgs &t, int64_t score_grid, int pages, hipStream_t stream)
{
    const int pick_grid = t.n_queries * t.a.kv.n_heads;
    if (score_grid > 0) {
        if (t.a.max_q == 1) hx_top_score_kernel<Q, E, D, true><<<(int)score_grid, TOP_THREADS, 0, stream>>>(t);
        else hx_top_score_kernel<Q, E, D, false><<<(int)score_grid, TOP_THREADS, 0, stream>>>(t);
    }
    const int cache = pages < 1024 ? pages : pages <= 2048 ? 2048 : 4096, lds = cache * 8;
    if (pages <= 256) hx_top_pick_kernel<Q, E, D, 64><<<pick_grid, 64, lds, stream>>>(t, cache);
    else hx_top_pick_kernel<Q, E, D, 512><<<pick_grid, 512, lds, stream>>>(t, cache);
}

template <typename Q, typename E>
void by_dim(const TopArgs &t, int64_t score_grid, int pages, hipStream_t stream)
{
    if (t.a.kv.dim == 64) score_and_pick<Q, E, 64>(t, score_grid, pages, stream);
    else if (t.a.kv.dim == 128) score_and_pick<Q, E, 128>(t, score_grid, pages, stream);
    else score_and_pick<Q, E, 256>(t, score_grid, pages, stream);
}

}  // namespace

extern "C" int hx_attend_top(hx_ctx *ctx, const hx_kv_pool *pool, int32_t layer, const hx_kv_seqs *seqs,
                             const hx_attend_args *args, const hx_top *top, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    KvView kv;
    bool any;
    if (int rc = hx_kv_view(ctx, pool, seqs, &kv)) return rc;
    if (int rc = hx_attend_check(ctx, pool, layer, kv, args, true, &any)) return rc;
    HX_REQUIRE(ctx, top, HX_ERR_INVALID_ARG, "NULL arguments");
    HX_REQUIRE(ctx, args->window == 0 && !args->parent, HX_ERR_INVALID_ARG, "chosen pages go without a window and without a tree");
    HX_REQUIRE(ctx, top->n_first >= 0 && top->n_last >= 1, HX_ERR_INVALID_ARG, "%d first and %d last pages", top->n_first, top->n_last);
    HX_REQUIRE(ctx, top->n_pages >= 1 && (int64_t)top->n_first + top->n_last <= top->n_pages, HX_ERR_INVALID_ARG, "%d pages for %d first and %d last", top->n_pages,
               top->n_first, top->n_last);
    HX_REQUIRE(ctx, top->n_pages <= HX_MAX_TOP, HX_ERR_SHAPE, "%d pages for a query, beyond %d", top->n_pages, HX_MAX_TOP);
    HX_REQUIRE(ctx, pool->bounds || kv.n_pages == 0, HX_ERR_INVALID_ARG, "a pool without bounds");
    if (!any) return HX_OK;
    const int H = kv.n_heads, n_q = args->n_q, n_pages = top->n_pages;
    const HxAttend whole = hx_attend_view(ctx, pool, layer, kv, *args);
    // no row has more pages than entries: no scores where all of them are seen
    const int64_t stride = kv.max_pages > n_pages && kv.n_pages > 0 ? ((int64_t)kv.max_pages + 15) / 16 * 16 : 0;
    const int picked_pages = kv.max_pages < 1 ? 1 : kv.max_pages < n_pages ? kv.max_pages : n_pages;
    const size_t line = (size_t)stride * (sizeof(double) + sizeof(float)) + (size_t)(stride / 16) * sizeof(float) + ((size_t)picked_pages + 1) * sizeof(int32_t);
    // so many queries at once that they stay below TOP_ROOM, and launches within their limits
    int64_t at_once = TOP_ROOM / (int64_t)(line * H);
    const int64_t tiles = (whole.group + 127) / 128, fits = hx_most_groups(1024) / (H * tiles * 64);
    HX_REQUIRE(ctx, fits > 0, HX_ERR_SHAPE, "%d query heads", whole.n_heads);
    at_once = at_once < fits ? at_once : fits;
    at_once = at_once < 1 ? 1 : at_once < n_q ? at_once : n_q;
    const int64_t q_tiles = (whole.max_q + 15) / 16, score_tiles = (int64_t)args->n * H * q_tiles;
    HX_REQUIRE(ctx, score_tiles <= hx_most_groups(TOP_THREADS), HX_ERR_SHAPE, "%d sequences of %d queries", args->n, whole.max_q);
    // Workgroups look at 64 pages at once, and again; as many of them for a tile of queries as there are pages for, up to 16 a CU in all (48 sequences over some 16000
    // tokens: 152 us, 156 with 8).
    int64_t about = ((int64_t)args->max_len >> kv.shift) + 1;
    about = about < stride ? about : stride;
    const int64_t useful = (about + 63) / 64, wanted = 16 * ctx->num_cu / score_tiles, most_chunks = hx_most_groups(TOP_THREADS) / score_tiles;
    int64_t chunks = useful < wanted ? useful : wanted;
    chunks = chunks < 1 ? 1 : chunks < most_chunks ? chunks : most_chunks;
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    const hipStream_t stream = (hipStream_t)stream_;
    const int64_t pairs = at_once * H;
    const size_t bytes = (size_t)pairs * line;
    if (int rc = hx_scratch(ctx, hx_serve(ctx)->top, bytes, stream)) return rc;
    const int64_t seen = (int64_t)n_pages << kv.shift, most = args->max_len < seen ? args->max_len : seen;
    auto part_of = [&](int64_t j, int64_t n) {
        HxAttend a = whole;
        a.n = a.n_q = (int)n;
        a.max_q = 1;
        a.picked_pages = picked_pages;
        a.q = (const char *)a.q + j * a.q_token * 2;
        a.out = (char *)a.out + j * a.out_token * 2;
        if (a.lse) a.lse += j * a.n_heads;
        return a;
    };
    // room for the parts of attention's keys too, before anything is launched: of a full part of the queries and of the last
    for (int64_t n : {at_once, n_q % at_once}) {
        if (n == 0) continue;
        HxAttend a = part_of(0, n);
        a.room_only = true;
        if (int rc = hx_attend_run(ctx, pool->dtype, args->dtype, a, (int)most, stream)) return rc;
    }
    TopArgs t{};
    t.a = whole;
    t.bounds = (const char *)pool->bounds + (int64_t)layer * kv.n_pages * hx_bounds_bytes(pool);
    t.n_pages = n_pages; t.picked_pages = picked_pages; t.n_first = top->n_first; t.n_last = top->n_last;
    t.stride = (int)stride;
    t.exact = (double *)hx_serve(ctx)->top.p;
    t.score = (float *)(t.exact + pairs * stride);
    t.off = t.score + pairs * stride;
    t.picked = (int32_t *)(t.off + pairs * (stride / 16));
    t.picked_len = t.picked + pairs * picked_pages;
    t.chosen = top->chosen;
    t.q_tiles = (int)q_tiles;
    t.chunks = (int)chunks;
    for (int64_t j = 0; j < n_q; j += at_once) {
        t.first_query = (int)j;
        t.n_queries = (int)(n_q - j < at_once ? n_q - j : at_once);
        const int64_t grid = stride ? score_tiles * chunks : 0;
        if (args->dtype == HX_BF16) by_dim<__bf16, __bf16>(t, grid, (int)about, stream);
        else if (pool->dtype == HX_F16) by_dim<_Float16, _Float16>(t, grid, (int)about, stream);
        else by_dim<_Float16, __bf16>(t, grid, (int)about, stream);
        if (int rc = hx_check_launch(ctx, "hx_top_pick_kernel")) return rc;
        HxAttend a = part_of(j, t.n_queries);
        a.picked = t.picked; a.picked_len = t.picked_len;
        if (int rc = hx_attend_run(ctx, pool->dtype, args->dtype, a, (int)most, stream)) return rc;
    }
    return HX_OK;
}
