// Rows cut to a budget of tokens by the weight that attention has given them.
//
// Four launches: each row's tokens that stay (a workgroup a row), the pages that rows need (one workgroup, so that they go out in the order of the
// rows), the moves, the tables.  24 rows of some 3000 tokens cut to 1024, 32 layers of 8 heads of 128: 1417 us, of which the moves 1400 at 4.4 TB/s.  One
// row of 4 layers cut to 1000: 40 us = 15 + 4 + 13 + 4 and what lies between, chains of lookups and barriers.
#include "hx_kv_plan.hpp"
#include "hx_nth.hpp"

namespace {

constexpr int EV_THREADS = 512, EV_WAVES = EV_THREADS / HX_WAVE;
constexpr int EV_CACHE = 8192;              // tokens of a row whose weights are kept in LDS
constexpr int EV_FULL = 2;                 // workgroups a CU from which the move is not divided further
constexpr int EV_AHEAD = 8;                // tokens that a thread moves at once

struct EvictArgs {
    KvView kv;
    KvPlanes planes;
    int n, n_keep, n_first, n_last, keep_pages;      // n_keep: no more than a row can have
    int slices;              // of a token's bytes, in the move
    const int32_t *row;
    float *weight;
    int64_t pitch;           // of a row's weights
    int32_t *kept;           // [n][kept_pitch] positions of the tokens that stay, then -1
    uint32_t kept_pitch;     // what the caller said, where it has asked for them
    int32_t *stay;           // [n] how many, -1: the row is left as it is
    int32_t *moves;          // [n] the first of them that changes its place, or all
    int32_t *need;           // [n] pages that are replaced
    int32_t *first;          // [n] pages that the rows before replace
    int32_t *fresh;          // [n][keep_pages] which of the row's new pages an entry gets, -1: it keeps its own
    int32_t *list;           // free pages
};

// Row i's kept positions from `from` on are none.  (No sign: the loop counts on past its end by a workgroup's threads, which may be near INT32_MAX.)
__device__ __forceinline__ void kept_none(const EvictArgs &a, int i, uint32_t from)
{
    int32_t *kept = a.kept + (int64_t)i * a.kept_pitch;
    for (uint32_t j = from + threadIdx.x; j < a.kept_pitch; j += EV_THREADS) kept[j] = -1;
}

// what is not above 0 counts as 0; keys of 0 are none, so that all are one up
__device__ __forceinline__ uint32_t weight_key(float w) { return (w > 0.0f ? __float_as_uint(w) : 0) + 1; }

// The threads before this one for which x is true, and *all of them.  s: EV_WAVES words.
__device__ __forceinline__ int count_before(bool x, int *s, int *all)
{
    const int lane = threadIdx.x & (HX_WAVE - 1), wave = threadIdx.x / HX_WAVE;
    const unsigned long long m = __builtin_amdgcn_ballot_w64(x);
    __syncthreads();
    if (lane == 0) s[wave] = __builtin_popcountll(m);
    __syncthreads();
    int before = __builtin_popcountll(m & ((1ull << lane) - 1)), total = 0;
#pragma unroll
    for (int w = 0; w < EV_WAVES; ++w) { const int c = s[w]; before += w < wave ? c : 0; total += c; }
    *all = total;
    return before;
}

__global__ __launch_bounds__(EV_THREADS) void hx_kv_evict_select_kernel(EvictArgs a)
{
    __shared__ NthState<uint32_t, EV_THREADS> s;
    __shared__ int s_count[EV_WAVES], s_count2[EV_WAVES];
    __shared__ uint32_t s_key[EV_CACHE];
    const KvView &kv = a.kv;
    const int i = blockIdx.x, tid = threadIdx.x, r = a.row[i];
    bool bad = r < 0 || r >= kv.rows;
    for (int j = tid; j < i; j += EV_THREADS) bad |= a.row[j] == r;
    bad = __syncthreads_or(bad);
    const int len = bad ? 0 : kv.len[r];
    bad = bad || !hx_row_ok(kv, r, len);
    int32_t *kept = a.kept + (int64_t)i * a.kept_pitch;
    if (bad || len <= a.n_keep) {
        if (bad && tid == 0) hx_raise(kv.status, HX_ERR_INDEX);
        kept_none(a, i, 0);
        if (tid == 0) { a.stay[i] = -1; a.need[i] = 0; }
        return;
    }
    const int32_t *table = hx_row(kv, r);
    const float *weight = a.weight + r * a.pitch;
    auto there = [&](int y) { const int page = table[y >> kv.shift]; return page >= 0 && page < kv.n_pages; };
    // 0: no page is there
    auto look = [&](int y) { return there(y) ? weight_key(weight[y]) : 0; };
    const bool cached = len <= EV_CACHE;
    if (cached) {
#pragma unroll 4
        for (int y = tid; y < len; y += EV_THREADS) s_key[y] = look(y);
        __syncthreads();
    }
    auto key_at = [&](int y) { return cached ? s_key[y] : look(y); };
    const int from = a.n_first, to = len - a.n_last;              // n_first + n_last <= n_keep < len
    int fixed = 0, all;
    for (int y0 = 0; y0 < a.n_first + a.n_last; y0 += EV_THREADS) {
        const int y = y0 + tid;
        count_before(y < a.n_first + a.n_last && key_at(y < a.n_first ? y : to + y - a.n_first) != 0, s_count, &all);
        fixed += all;
    }
    const int want = a.n_keep - fixed;
    uint32_t edge = ~0u;
    int equals = 0;
    if (want > 0) {
        nth_largest(key_at, from, to, want, s);
        edge = s.edge;
        equals = s.equals;
    }
    // the tokens that stay, in order
    int n = 0, same = 0, moves = INT32_MAX;
    for (int y0 = 0; y0 < len; y0 += EV_THREADS) {
        const int y = y0 + tid;
        const uint32_t key = y < len ? key_at(y) : 0;
        const bool here = key != 0, between = y >= from && y < to;
        const uint32_t x = between ? key : 0;
        const bool equal = x == edge && x > 0;
        const int rank = same + count_before(equal, s_count, &all);
        same += all;
        const bool take = here && (!between || x > edge || (equal && rank < equals));
        const int at = n + count_before(take, s_count2, &all);
        n += all;
        if (take) {
            kept[at] = y;
            if (y != at && at < moves) moves = at;
        }
    }
    kept_none(a, i, n);
    for (int b = tid; b < hx_pages_of(len, kv.shift); b += EV_THREADS)
        if (table[b] >= kv.n_pages) hx_raise(kv.status, HX_ERR_INDEX);
#pragma unroll
    for (int d = HX_WAVE / 2; d > 0; d >>= 1) { const int o = __shfl_xor(moves, d); moves = o < moves ? o : moves; }
    __syncthreads();
    if ((tid & (HX_WAVE - 1)) == 0) s_count[tid / HX_WAVE] = moves;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < EV_WAVES; ++w) moves = s_count[w] < moves ? s_count[w] : moves;
    moves = moves < n ? moves : n;
    // Entries in which something changes, and the one that the row goes on in, which ends with them: they have to be this row's alone.
    const int pages = hx_pages_of(n, kv.shift);
    int need = 0;
    for (int b0 = moves >> kv.shift; b0 < pages; b0 += EV_THREADS) {
        const int b = b0 + tid, page = b < pages ? table[b] : -1;
        const bool own = page >= 0 && page < kv.n_pages && kv.ref[page] <= 1;
        const int rank = need + count_before(b < pages && !own, s_count, &all);
        need += all;
        if (b < pages) a.fresh[(int64_t)i * a.keep_pages + b] = own ? -1 : rank;
    }
    for (int b = tid; b < moves >> kv.shift && b < pages; b += EV_THREADS) a.fresh[(int64_t)i * a.keep_pages + b] = -1;
    if (tid == 0) { a.stay[i] = n; a.moves[i] = moves; a.need[i] = need; }
}

__global__ __launch_bounds__(PL_THREADS) void hx_kv_evict_plan_kernel(EvictArgs a)
{
    __shared__ int64_t s[PL_WAVES];
    const KvView &kv = a.kv;
    int64_t want = 0;
    for (int i0 = 0; i0 < a.n; i0 += PL_THREADS) {
        const int i = i0 + threadIdx.x, need = i < a.n ? a.need[i] : 0;
        int64_t all;
        const int64_t before = want + block_before(need, s, &all);
        if (i < a.n) a.first[i] = (int)(before < INT32_MAX ? before : INT32_MAX);
        want += all;
    }
    if (want == 0) return;
    const int found = first_pages<false>(kv.ref, 0, kv.n_pages, want < kv.n_pages ? (int)want : kv.n_pages, a.list, s);
    for (int i = threadIdx.x; i < a.n; i += PL_THREADS) {
        if (a.need[i] == 0 || (int64_t)a.first[i] + a.need[i] <= found) continue;
        hx_raise(kv.status, HX_ERR_CAPACITY);
        a.stay[i] = -1;
    }
    __syncthreads();
    for (uint32_t j = threadIdx.x; j < (uint32_t)found; j += PL_THREADS) {
        int lo = 0, hi = a.n - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if ((uint32_t)a.first[mid] <= j) lo = mid; else hi = mid - 1;
        }
        if ((int64_t)a.first[lo] + a.need[lo] <= found) kv.ref[a.list[j]] = 1;
    }
}

// A row's entry after the call.
__device__ __forceinline__ int page_after(const EvictArgs &a, int i, int b, const int32_t *table)
{
    const int f = a.fresh[(int64_t)i * a.keep_pages + b];
    return f < 0 ? table[b] : a.list[a.first[i] + f];
}

// Workgroup (i, part): a head of one array of a layer, of few such a slice of its tokens' bytes, or, first, the row's weights.  Tokens move to lower positions, in order: a round's tokens are all
// loaded before any of them is stored, and later rounds load only what lies behind what has been stored.
__global__ __launch_bounds__(EV_THREADS) void hx_kv_evict_move_kernel(EvictArgs a)
{
    const KvView &kv = a.kv;
    const int heads = kv.n_heads, parts = 1 + a.planes.n * kv.n_layers * heads * a.slices, i = blockIdx.x / parts, part = blockIdx.x % parts, tid = threadIdx.x;
    const int n = a.stay[i], r = a.row[i];
    if (n < 0) return;
    const int32_t *kept = a.kept + (int64_t)i * a.kept_pitch;
    const int begin = a.moves[i];
    if (part == 0) {
        float *w = a.weight + r * a.pitch;
        for (int j0 = begin; j0 < n; j0 += EV_THREADS * EV_AHEAD) {
            float x[EV_AHEAD];
#pragma unroll
            for (int k = 0; k < EV_AHEAD; ++k) {
                const int j = j0 + k * EV_THREADS + tid;
                if (j < n) x[k] = w[kept[j]];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < EV_AHEAD; ++k) {
                const int j = j0 + k * EV_THREADS + tid;
                if (j < n) w[j] = x[k];
            }
        }
        __syncthreads();
        for (int y = n + tid; y < kv.len[r]; y += EV_THREADS) w[y] = 0.0f;
        return;
    }
    const int32_t *table = hx_row(kv, r);
    const int slice = (part - 1) % a.slices, p = (part - 1) / a.slices, head = p % heads, which = p / heads % a.planes.n, layer = p / heads / a.planes.n, in_page = (1 << kv.shift) - 1;
    const Plane x = plane(a.planes, which);
    const int64_t head_bytes = (int64_t)x.row_bytes << kv.shift;
    char *at = x.at + ((int64_t)layer * kv.n_pages * heads + head) * head_bytes;
    // pages that are replaced are replaced whole: their tokens that keep their places are copied too
    const int start = begin & ~in_page;
    by_width(x.row_bytes, [&](auto unit) {
        using U = decltype(unit);
        const int all = x.row_bytes / (int)sizeof(U), c0 = all * slice / a.slices, pieces = all * (slice + 1) / a.slices - c0;       // (at most 128)
        if (pieces == 0) return;
        const int slots = EV_THREADS / pieces, slot = tid / pieces, c = c0 + tid % pieces;
        for (int j0 = start; j0 < n; j0 += slots * EV_AHEAD) {
            U y[EV_AHEAD];
            int64_t to[EV_AHEAD];
#pragma unroll
            for (int k = 0; k < EV_AHEAD; ++k) {
                const int at_k = j0 + k * slots + slot, j = slot < slots && at_k < n ? at_k : j0;
                const int from = kept[j], old = table[from >> kv.shift], page = page_after(a, i, j >> kv.shift, table);
                const bool moves = at_k == j && (from != j || page != old);
                to[k] = moves ? (int64_t)page * heads * head_bytes + (int64_t)(j & in_page) * x.row_bytes + c * sizeof(U) : -1;
                y[k] = *(const U *)(at + (int64_t)old * heads * head_bytes + (int64_t)(from & in_page) * x.row_bytes + c * sizeof(U));
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < EV_AHEAD; ++k)
                if (to[k] >= 0) *(U *)(at + to[k]) = y[k];
        }
    });
}

__global__ __launch_bounds__(EV_THREADS) void hx_kv_evict_apply_kernel(EvictArgs a)
{
    const KvView &kv = a.kv;
    const int i = blockIdx.x, n = a.stay[i], r = a.row[i];
    if (n < 0) {
        kept_none(a, i, 0);
        return;
    }
    int32_t *table = hx_row(kv, r);
    const int len = kv.len[r], pages = hx_pages_of(n, kv.shift);
    for (int b = threadIdx.x; b < hx_pages_of(len, kv.shift); b += EV_THREADS) {
        const int old = table[b], now = b < pages ? page_after(a, i, b, table) : -1;
        if (now == old) continue;
        table[b] = now;
        if (old >= 0) give_back(kv, old);
    }
    __syncthreads();
    if (threadIdx.x == 0) kv.len[r] = n;
}

}  // namespace

extern "C" int hx_kv_evict(hx_ctx *ctx, const hx_kv_pool *pool, const hx_kv_seqs *seqs, int32_t n, const int32_t *row,
                           float *weight, int32_t n_keep, int32_t n_first, int32_t n_last, int32_t *kept, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    KvView kv;
    if (int rc = hx_kv_view(ctx, pool, seqs, &kv)) return rc;
    HX_REQUIRE(ctx, n >= 0, HX_ERR_INVALID_ARG, "negative size");
    HX_REQUIRE(ctx, n_keep >= 1 && n_first >= 0 && n_last >= 0 && (int64_t)n_first + n_last <= n_keep, HX_ERR_INVALID_ARG, "%d tokens for %d first and %d last",
               n_keep, n_first, n_last);
    if (n == 0) return HX_OK;
    HX_REQUIRE(ctx, row && weight, HX_ERR_INVALID_ARG, "NULL array");
    HX_REQUIRE(ctx, ((uintptr_t)weight & 3) == 0, HX_ERR_INVALID_ARG, "weights are not aligned to their type");
    HX_REQUIRE(ctx, !seqs->weight || seqs->weight == weight, HX_ERR_INVALID_ARG, "weights that are not the sequences' own, which would stay in their old places");
    HX_REQUIRE(ctx, kv.rows > 0, HX_ERR_INVALID_ARG, "%d rows asked for of no sequences", n);
    const KvPlanes planes = hx_kv_planes(pool);
    // a round is a chain of lookups, and a slice of half the bytes takes twice the tokens in one: slices until the chip is full, of no less than 64 bytes.
    int slices = 1;
    while (2 * (int64_t)n * planes.n * kv.n_layers * kv.n_heads * slices <= EV_FULL * ctx->num_cu && planes.row_bytes[0] >= 128 * slices) slices *= 2;
    const int64_t parts = 1 + (int64_t)planes.n * kv.n_layers * kv.n_heads * slices;
    HX_REQUIRE(ctx, n * parts <= hx_most_groups(EV_THREADS), HX_ERR_SHAPE, "%d rows of %d layers of %d heads in one call", n, kv.n_layers, kv.n_heads);
    HX_REQUIRE(ctx, (int64_t)kv.max_pages << kv.shift <= INT32_MAX / 2, HX_ERR_SHAPE, "%d pages of %d tokens a row", kv.max_pages, 1 << kv.shift);
    // a budget beyond what a row can have needs no more room than that
    const int pitch = kv.max_pages << kv.shift, most = n_keep < pitch ? n_keep : pitch, keep_pages = hx_pages_of(most, kv.shift);
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    const hipStream_t stream = (hipStream_t)stream_;
    const size_t words = (size_t)n * (4 + (size_t)keep_pages + (kept ? 0 : (size_t)most)) + kv.n_pages;
    if (int rc = hx_scratch(ctx, hx_serve(ctx)->kv, words * sizeof(int32_t), stream)) return rc;
    int32_t *w = (int32_t *)hx_serve(ctx)->kv.p;
    const size_t N = n;
    EvictArgs a{kv, planes, n, most, n_first, n_last, keep_pages, slices, row, weight, pitch,
                kept ? kept : w + N * (4 + (size_t)keep_pages) + kv.n_pages, (uint32_t)(kept ? n_keep : most), w, w + N, w + 2 * N, w + 3 * N, w + 4 * N, w + N * (4 + (size_t)keep_pages)};
    hx_kv_evict_select_kernel<<<n, EV_THREADS, 0, stream>>>(a);
    hx_kv_evict_plan_kernel<<<1, PL_THREADS, 0, stream>>>(a);
    hx_kv_evict_move_kernel<<<(int)(n * parts), EV_THREADS, 0, stream>>>(a);
    hx_kv_evict_apply_kernel<<<n, EV_THREADS, 0, stream>>>(a);
    return hx_check_launch(ctx, "hx_kv_evict_apply_kernel");
}
