// Attention over the pages that every query chooses for every KV head: what a page's keys can score at most, the pages of the largest of these,
// and hx_attend's kernels over them, for which each query and KV head is a sequence with a table of its own.
#include "hx_attend_common.hpp"
#include "hx_nth.hpp"

namespace {

constexpr int TOP_THREADS = 256;
constexpr int64_t TOP_SCORES = (int64_t)1 << 28;         // bytes of scores at once

struct TopArgs {
    AttendArgs a;
    const void *bounds;              // of the layer
    int first_query, n_queries;      // of this part of the call
    int n_pages, n_first, n_last;
    int stride;                      // entries of a row
    double *score;                   // [query][KV head][stride], NULL where no row has more than n_pages entries
    int32_t *picked, *picked_len;    // what hx_attend's kernels read
    int32_t *chosen;                 // of the call's first query, or NULL
    int chunks;                      // workgroups that look at the pages of one query and KV head
};

// A query's row: its pages up to its own, `own`.
struct Place {
    bool ok;
    int pos, own;
    const int32_t *table;
};
__device__ __forceinline__ Place place(const AttendArgs &a, int j)
{
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.q_ptr[mid] <= j) lo = mid; else hi = mid - 1;
    }
    const Seq s = sequence(a, lo * a.kv.n_heads);
    Place p;
    p.ok = s.ok && j >= s.q0 && j < s.q0 + s.nq;
    p.pos = p.ok ? s.base + j - s.q0 : 0;
    p.own = p.pos >> a.kv.shift;
    p.table = s.table;
    return p;
}

// ---- what a page can score ---------------------------------------------------

__device__ __forceinline__ double across(double x, int d)
{
    const uint64_t v = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __shfl_xor((uint32_t)v, d), hi = __shfl_xor((uint32_t)(v >> 32), d);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Four heads' sums over LANES lanes, and the largest: half of the heads is given away for each of the first two steps.  Heads from `heads` on have
// none.  *odd: whether any of them is NaN.
template <int LANES>
__device__ __forceinline__ double largest_sum(const double *v, int sub, int heads, bool *odd)
{
    const bool up = sub & (LANES / 2), up2 = sub & (LANES / 4);
    double x0 = up ? v[2] : v[0], x1 = up ? v[3] : v[1];
    x0 += across(up ? v[0] : v[2], LANES / 2);
    x1 += across(up ? v[1] : v[3], LANES / 2);
    double x = (up2 ? x1 : x0) + across(up2 ? x0 : x1, LANES / 4);
#pragma unroll
    for (int d = LANES / 8; d > 0; d >>= 1) x += across(x, d);
    if ((up ? 2 : 0) + (up2 ? 1 : 0) >= heads) x = -__builtin_inf();
    *odd = x != x;
    x = fmax(x, across(x, LANES / 4));
    return fmax(x, across(x, LANES / 2));
}

// Bounds of E, queries of Q.  A page's bounds lie over D / 8 lanes, 8 places each.  A product of two 16-bit numbers is exact in 64 bits, and the sums are off by some 2^-50 of
// their terms: which of two pages comes first does not go by how they are added, but for differences below that.
template <typename Q, typename E, int D>
__global__ __launch_bounds__(TOP_THREADS) void hx_top_score_kernel(TopArgs t)
{
    using Q8 = typename Types<Q>::x8;
    using E8 = typename Types<E>::x8;
    constexpr int LANES = D / 8, PER = 64 / LANES, STEPS = 4, WAVES = TOP_THREADS / 64;      // pages a wavefront has at once, how many times
    const AttendArgs &a = t.a;
    const KvView &kv = a.kv;
    const int pairs = t.n_queries * kv.n_heads, pair = blockIdx.x % pairs, head = pair % kv.n_heads, j = t.first_query + pair / kv.n_heads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % LANES, slot = lane / LANES;
    const Place p = place(a, j);
    if (!p.ok || p.own < t.n_pages) return;                       // (no more pages than it may see)
    const int last = p.own - t.n_last;
    for (int chunk = blockIdx.x / pairs;; chunk += t.chunks) {
        const int b0 = t.n_first + (chunk * WAVES + wave) * (STEPS * PER) + slot;
        if (t.n_first + chunk * WAVES * (STEPS * PER) > last) break;
        E8 lo[STEPS], hi[STEPS];
        int page[STEPS];
        double best[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int b = b0 + s * PER;
            page[s] = in_pool(kv, b <= last ? p.table[b] : -1);
            const E *at = (const E *)t.bounds + ((int64_t)(page[s] < 0 ? 0 : page[s]) * kv.n_heads + head) * (2 * D) + sub * 8;
            lo[s] = *(const E8 *)at;
            hi[s] = *(const E8 *)(at + D);
            best[s] = -__builtin_inf();
        }
        for (int g0 = 0; g0 < a.group; g0 += 4) {
            double above[4][8], below[4][8];                      // the query's numbers where they are not below 0, and where they are
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int qhead = head * a.group + (g0 + g < a.group ? g0 + g : g0);
                const Q *q = (const Q *)a.q + (int64_t)j * a.q_token + (int64_t)qhead * a.q_head + sub * 8;
                Q8 x;
                if (a.q_wide) x = *(const Q8 *)q;
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = q[i];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const double y = a.scale < 0 ? -(double)(float)x[i] : (double)(float)x[i];
                    above[g][i] = y >= 0 ? y : y < 0 ? 0.0 : y;
                    below[g][i] = y < 0 ? y : 0.0;
                }
            }
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                double v[4] = {};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const double l = (double)(float)lo[s][i], h = (double)(float)hi[s][i];
#pragma unroll
                    for (int g = 0; g < 4; ++g) v[g] = fma(below[g][i], l, fma(above[g][i], h, v[g]));
                }
                bool odd;
                double x = largest_sum<LANES>(v, sub, a.group - g0, &odd);
                if (__builtin_amdgcn_ballot_w64(odd)) {
                    // 0 times an infinite bound is NaN; the bound that does not count is left out then
#pragma unroll
                    for (int g = 0; g < 4; ++g) v[g] = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const bool under = below[g][i] < 0;
                            v[g] = fma(under ? below[g][i] : above[g][i], (double)(float)(under ? lo[s][i] : hi[s][i]), v[g]);
                        }
                    x = largest_sum<LANES>(v, sub, a.group - g0, &odd);
                    // a bound that is NaN is taken for +infinity, whichever of the lanes has seen it
                    const unsigned long long any = __builtin_amdgcn_ballot_w64(odd);
                    const unsigned long long mine = LANES == 64 ? ~0ull : ((1ull << LANES) - 1) << (slot * LANES);
                    if (any & mine) x = __builtin_inf();
                }
                best[s] = fmax(best[s], x);
            }
        }
        if (sub == 0)
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int b = b0 + s * PER;
                if (b <= last) t.score[(int64_t)pair * t.stride + b] = page[s] < 0 ? -__builtin_inf() : best[s];
            }
    }
}

// ---- the pages of the largest ------------------------------------------------

constexpr int PICK_WAVES = TOP_THREADS / 64;

// A score's key, 0 where it is -infinity (-0 and 0 are the same number).
__device__ __forceinline__ uint64_t key_of(double x) { return x == -__builtin_inf() ? 0 : nth_key(x + 0.0); }

// A workgroup a query and KV head.
__global__ __launch_bounds__(TOP_THREADS) void hx_top_pick_kernel(TopArgs t)
{
    __shared__ NthState<uint64_t, TOP_THREADS> s;
    __shared__ int s_before[2][PICK_WAVES];
    const AttendArgs &a = t.a;
    const KvView &kv = a.kv;
    const int pair = blockIdx.x, head = pair % kv.n_heads, j = t.first_query + pair / kv.n_heads;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Place p = place(a, j);
    int32_t *picked = t.picked + (int64_t)pair * t.n_pages;
    int32_t *chosen = t.chosen ? t.chosen + ((int64_t)j * kv.n_heads + head) * t.n_pages : nullptr;
    if (!p.ok) {
        if (tid == 0) { hx_raise(kv.status, HX_ERR_INDEX); picked[0] = -1; t.picked_len[pair] = 1; }
        if (chosen)
            for (int i = tid; i < t.n_pages; i += TOP_THREADS) chosen[i] = -1;
        return;
    }
    const bool all = p.own < t.n_pages || kv.n_pages == 0;
    const int from = t.n_first, to = p.own - t.n_last + 1;         // the pages between those that are seen in any case
    const double *score = t.score + (int64_t)pair * t.stride;
    uint64_t edge = 0;
    int equals = 0;
    if (!all) {
        int want = t.n_pages;
        int fixed = 0;
        for (int i = tid; i < t.n_first + t.n_last; i += TOP_THREADS) {
            const int page = p.table[i < t.n_first ? i : p.own - t.n_last + 1 + i - t.n_first];
            fixed += page >= 0 && page < kv.n_pages;
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) fixed += __shfl_xor(fixed, d);
        if (lane == 0) s_before[0][wave] = fixed;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < PICK_WAVES; ++w) want -= s_before[0][w];
        __syncthreads();
        if (want > 0) {
            nth_largest([&](int b) { return key_of(score[b]); }, from, to, want, s);
            edge = s.edge;
            equals = s.equals;
        } else edge = ~0ull;
    }
    // the pages in rising order
    int n = 0, seen_equal = 0;
    for (int b0 = 0; b0 <= p.own; b0 += TOP_THREADS) {
        const int b = b0 + tid;
        const int page = in_pool(kv, b <= p.own ? p.table[b] : -1);
        const bool between = !all && b >= from && b < to;
        const uint64_t x = between && page >= 0 ? key_of(score[b]) : 0;
        const bool equal = x == edge && x > 0;
        const unsigned long long e = __builtin_amdgcn_ballot_w64(equal);
        if (lane == 0) s_before[0][wave] = __builtin_popcountll(e);
        __syncthreads();
        int rank = seen_equal + __builtin_popcountll(e & ((1ull << lane) - 1)), all_equal = 0;
#pragma unroll
        for (int w = 0; w < PICK_WAVES; ++w) { rank += w < wave ? s_before[0][w] : 0; all_equal += s_before[0][w]; }
        const bool take = page >= 0 && (!between || x > edge || (equal && rank < equals));
        const unsigned long long m = __builtin_amdgcn_ballot_w64(take);
        if (lane == 0) s_before[1][wave] = __builtin_popcountll(m);
        __syncthreads();
        int at = n + __builtin_popcountll(m & ((1ull << lane) - 1));
#pragma unroll
        for (int w = 0; w < PICK_WAVES; ++w) { at += w < wave ? s_before[1][w] : 0; n += s_before[1][w]; }
        seen_equal += all_equal;
        if (take) {
            picked[at] = page;
            if (chosen) chosen[at] = b;
            // where its own page is there it is the last of all; else all that are chosen are full
            if (b == p.own) t.picked_len[pair] = (at << kv.shift) + (p.pos & ((1 << kv.shift) - 1)) + 1;
        }
        __syncthreads();
    }
    if (chosen)
        for (int i = n + tid; i < t.n_pages; i += TOP_THREADS) chosen[i] = -1;
    const int own_page = p.table[p.own];
    if (tid == 0 && (own_page < 0 || own_page >= kv.n_pages)) {
        if (n == 0) picked[0] = -1;
        t.picked_len[pair] = n == 0 ? 1 : n << kv.shift;
    }
}

template <typename Q, typename E>
void score(const TopArgs &t, int64_t grid, hipStream_t stream)
{
    if (t.a.kv.dim == 64) hx_top_score_kernel<Q, E, 64><<<(int)grid, TOP_THREADS, 0, stream>>>(t);
    else if (t.a.kv.dim == 128) hx_top_score_kernel<Q, E, 128><<<(int)grid, TOP_THREADS, 0, stream>>>(t);
    else hx_top_score_kernel<Q, E, 256><<<(int)grid, TOP_THREADS, 0, stream>>>(t);
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
    const int H = kv.n_heads, n_q = args->n_q;
    // more pages than any row has are never chosen
    const int n_pages = top->n_pages;
    const int64_t stride = kv.max_pages > n_pages ? kv.max_pages : 0;
    // so many queries at once that scores stay below TOP_SCORES, and launches within their limits
    const HxAttend whole = hx_attend_view(ctx, pool, layer, kv, *args);
    int64_t at_once = stride ? TOP_SCORES / (stride * H * (int64_t)sizeof(double)) : n_q;
    const int64_t tiles = (whole.group + 127) / 128, fits = hx_most_groups(TOP_THREADS) / (H * tiles * 64);
    HX_REQUIRE(ctx, fits > 0, HX_ERR_SHAPE, "%d query heads", whole.n_heads);
    at_once = at_once < fits ? at_once : fits;
    at_once = at_once < 1 ? 1 : at_once < n_q ? at_once : n_q;
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    const hipStream_t stream = (hipStream_t)stream_;
    const int64_t pairs = at_once * H;
    const size_t bytes = (size_t)pairs * (stride * sizeof(double) + ((size_t)n_pages + 1) * sizeof(int32_t));
    if (int rc = hx_scratch(ctx, hx_serve(ctx)->top, bytes, stream)) return rc;
    const int64_t seen = (int64_t)n_pages << kv.shift, most = args->max_len < seen ? args->max_len : seen;
    auto part_of = [&](int64_t j, int64_t n) {
        HxAttend a = whole;
        a.n = a.n_q = (int)n;
        a.max_q = 1;
        a.picked_pages = n_pages;
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
    t.n_pages = n_pages; t.n_first = top->n_first; t.n_last = top->n_last;
    t.stride = (int)stride;
    t.score = (double *)hx_serve(ctx)->top.p;
    t.picked = (int32_t *)(t.score + pairs * stride);
    t.picked_len = t.picked + pairs * n_pages;
    t.chosen = top->chosen;
    const int per = TOP_THREADS / (kv.dim / 8) * 4;                 // pages that a workgroup looks at at once
    const int64_t about = ((int64_t)args->max_len >> kv.shift) + 1, chunks = ((about < stride ? about : stride) + per - 1) / per;
    t.chunks = (int)(chunks < 1 ? 1 : chunks < 64 ? chunks : 64);
    for (int64_t j = 0; j < n_q; j += at_once) {
        t.first_query = (int)j;
        t.n_queries = (int)(n_q - j < at_once ? n_q - j : at_once);
        const int64_t now = (int64_t)t.n_queries * H;
        if (stride && kv.n_pages > 0) {
            const int64_t grid = now * t.chunks;
            const bool bf16 = args->dtype == HX_BF16;
            if (bf16) score<__bf16, __bf16>(t, grid, stream);
            else if (pool->dtype == HX_F16) score<_Float16, _Float16>(t, grid, stream);
            else score<_Float16, __bf16>(t, grid, stream);
            if (int rc = hx_check_launch(ctx, "hx_top_score_kernel")) return rc;
        }
        hx_top_pick_kernel<<<(int)now, TOP_THREADS, 0, stream>>>(t);
        if (int rc = hx_check_launch(ctx, "hx_top_pick_kernel")) return rc;
        HxAttend a = part_of(j, t.n_queries);
        a.picked = t.picked; a.picked_len = t.picked_len;
        if (int rc = hx_attend_run(ctx, pool->dtype, args->dtype, a, (int)most, stream)) return rc;
    }
    return HX_OK;
}
