// Pages of a decode instance's cache: fork, grow, write, keep, free, compact.
//
// Everything here is integers and copies; results depend on the arguments alone.  Which pages a call takes is decided by one
// workgroup that looks through `ref` from its start (the free pages of lowest number, in the order of the call's rows), and the
// copying is spread over the chip.  Counters of entries and pages have no sign: they pass a limit of INT32_MAX by a workgroup's threads.
#include "hx_serve.hpp"

namespace {

constexpr int PL_THREADS = 1024;           // the planning workgroup
constexpr int PL_WAVES = PL_THREADS / HX_WAVE;
constexpr int CP_THREADS = 256;            // workgroups that copy
constexpr int NO_CLAIM = 0x7fffffff;

// Sum of x over the workgroup's threads before this one; *all = over all of them.  s: PL_WAVES words.
__device__ __forceinline__ int64_t block_before(int64_t x, int64_t *s, int64_t *all)
{
    const int lane = threadIdx.x & (HX_WAVE - 1), w = threadIdx.x / HX_WAVE;
    int64_t sum = x;
#pragma unroll
    for (int d = 1; d < HX_WAVE; d <<= 1) {
        const int64_t y = __shfl_up(sum, d);
        if (lane >= d) sum += y;
    }
    __syncthreads();
    if (lane == HX_WAVE - 1) s[w] = sum;
    __syncthreads();
    int64_t before = 0, total = 0;
#pragma unroll
    for (int i = 0; i < PL_WAVES; ++i) {
        const int64_t y = s[i];
        before += i < w ? y : 0;
        total += y;
    }
    *all = total;
    return before + sum - x;
}

// The first `want` pages that are free, ref <= 0 (USED: in use), from page `from` on and before `to`, into list; returns how many there are, at most `want`.
// A wavefront looks at 8 x 64 neighbouring pages at a time, the workgroup at 8192.
constexpr int SCAN_EACH = 8;
template <bool USED>
__device__ int first_pages(const int32_t *ref, int from, int to, int want, int32_t *list, int64_t *s)
{
    const int lane = threadIdx.x & (HX_WAVE - 1), w = threadIdx.x / HX_WAVE;
    int found = 0;
    for (int64_t at = from; at < to && found < want; at += PL_THREADS * SCAN_EACH) {
        const int64_t mine = at + w * (HX_WAVE * SCAN_EACH) + lane;
        int r[SCAN_EACH];
#pragma unroll
        for (int j = 0; j < SCAN_EACH; ++j) r[j] = mine + j * HX_WAVE < to ? ref[mine + j * HX_WAVE] : (USED ? 0 : 1);
        unsigned long long m[SCAN_EACH];
        int count = 0;
#pragma unroll
        for (int j = 0; j < SCAN_EACH; ++j) {
            m[j] = __builtin_amdgcn_ballot_w64((r[j] > 0) == USED);
            count += __builtin_popcountll(m[j]);
        }
        int64_t all;
        // every lane counts its wavefront's pages, lane 0's share is what is added up
        int64_t before = block_before(lane == 0 ? count : 0, s, &all);
        before = __shfl(before, 0);
        int rank = found + (int)before;
#pragma unroll
        for (int j = 0; j < SCAN_EACH; ++j) {
            const int mine_rank = rank + __builtin_popcountll(m[j] & ((1ull << lane) - 1));
            if (((m[j] >> lane) & 1) && mine_rank < want) list[mine_rank] = (int32_t)(mine + j * HX_WAVE);
            rank += __builtin_popcountll(m[j]);
        }
        found += (int)all;
    }
    __syncthreads();
    return found < want ? found : want;
}

// Of several rows of a call with the same number the first counts.  claim: a word for each row of the tables.
__device__ void claim_rows(const int32_t *row, int n, int rows, int32_t *claim)
{
    for (int i = threadIdx.x; i < n; i += PL_THREADS)
        if (row[i] >= 0 && row[i] < rows) __hip_atomic_store(claim + row[i], NO_CLAIM, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += PL_THREADS)
        if (row[i] >= 0 && row[i] < rows) atomicMin(claim + row[i], i);
    __syncthreads();
}

struct ForkArgs {
    KvView kv;
    int n;
    const int32_t *src, *dst, *n_tok;
    int32_t *claim;          // [rows]
    int32_t *tok;            // [n] tokens of the copy, -1: none is made
    int32_t *from, *to;      // [n] the last page's, -1: none is copied
    int32_t *list;           // [n] free pages
    int row_bytes;           // of a token in one head
};

// One workgroup, so that pages go out in the order of the rows: a chain of memory round trips (the claim, the source's length and last
// page, the counts of 8192 pages at a time).  4 copies of one call: 7.4 us; 256 copies: 11.
__global__ __launch_bounds__(PL_THREADS) void hx_kv_fork_plan_kernel(ForkArgs a)
{
    __shared__ int64_t s[PL_WAVES];
    const KvView &kv = a.kv;
    claim_rows(a.dst, a.n, kv.rows, a.claim);
    bool bad = false;
    int need = 0;
    const int rounds = (a.n + PL_THREADS - 1) / PL_THREADS;
    for (int it = 0; it < rounds; ++it) {
        const int i = it * PL_THREADS + threadIdx.x;
        int t = -1, page = -1;
        if (i < a.n) {
            const int r = a.src[i], d = a.dst[i];
            const bool ok = r >= 0 && r < kv.rows && d >= 0 && d < kv.rows && r != d && hx_sync_load(a.claim + d) == i && kv.len[d] == 0;
            if (ok) {
                const int len = kv.len[r];
                t = a.n_tok ? a.n_tok[i] : len;
                if (t < 0 || t > len || !hx_row_ok(kv, r, len)) t = -1;
            }
            if (t < 0) bad = true;
            if (t > 0 && (t & ((1 << kv.shift) - 1))) {
                page = hx_row(kv, r)[t >> kv.shift];
                if (page >= kv.n_pages) { bad = true; page = -1; }
            }
        }
        int64_t all;
        const int rank = need + (int)block_before(t >= 0 && page >= 0, s, &all);
        if (i < a.n) {
            a.tok[i] = t;
            a.from[i] = t >= 0 && page >= 0 ? page : -1;
            a.to[i] = rank;                          // for now: which of the free pages
        }
        need += (int)all;
    }
    if (bad) hx_raise(kv.status, HX_ERR_INDEX);
    const int found = first_pages<false>(kv.ref, 0, kv.n_pages, need, a.list, s);
    for (int i = threadIdx.x; i < a.n; i += PL_THREADS) {
        const int t = a.tok[i];
        if (t < 0) continue;
        if (a.from[i] >= 0) {
            const int rank = a.to[i];
            if (rank >= found) {
                hx_raise(kv.status, HX_ERR_CAPACITY);
                a.tok[i] = a.from[i] = -1;
                continue;
            }
            const int page = a.list[rank];
            a.to[i] = page;
            kv.ref[page] = 1;
            hx_row(kv, a.dst[i])[t >> kv.shift] = page;
        }
        kv.len[a.dst[i]] = t;
    }
}

// Workgroup (i, 0): the shared pages of copy i; (i, 1 + 2 layer + v): its last page's tokens in one layer's keys or values, 16 bytes a
// thread.  Bound by HBM: 256 copies of tails in 32 layers, 1.0 GB read and written: 169 us, and their sources come from the caches three
// times of four (a plain copy reaches 4.7 TB/s).
__global__ __launch_bounds__(CP_THREADS) void hx_kv_fork_copy_kernel(ForkArgs a)
{
    const KvView &kv = a.kv;
    const int parts = 1 + 2 * kv.n_layers, i = blockIdx.x / parts, part = blockIdx.x % parts;
    const int t = a.tok[i];
    if (t <= 0) return;
    if (part == 0) {
        const int32_t *from = hx_row(kv, a.src[i]);
        int32_t *to = hx_row(kv, a.dst[i]);
        for (uint32_t b = threadIdx.x; b < (uint32_t)t >> kv.shift; b += CP_THREADS) {
            int page = from[b];
            if (page >= kv.n_pages) { hx_raise(kv.status, HX_ERR_INDEX); page = -1; }
            to[b] = page;
            if (page >= 0) atomicAdd(kv.ref + page, 1);
        }
        // a last page that the source has given back is none of the copy's either
        if (threadIdx.x == 0 && (t & ((1 << kv.shift) - 1)) && a.from[i] < 0) to[t >> kv.shift] = -1;
        return;
    }
    if (a.from[i] < 0) return;
    const int layer = (part - 1) >> 1, toks = t & ((1 << kv.shift) - 1);
    char *base = (char *)(((part - 1) & 1) ? kv.v : kv.k);
    const int64_t head_bytes = (int64_t)a.row_bytes << kv.shift;
    const char *from = base + ((int64_t)layer * kv.n_pages + a.from[i]) * kv.n_heads * head_bytes;
    char *to = base + ((int64_t)layer * kv.n_pages + a.to[i]) * kv.n_heads * head_bytes;
    const int per = toks * a.row_bytes / 16;                   // 16-byte pieces of a head
    for (int c = threadIdx.x; c < per * kv.n_heads; c += CP_THREADS) {
        const int64_t at = (c / per) * head_bytes + (int64_t)(c % per) * 16;
        *(uint4 *)(to + at) = *(const uint4 *)(from + at);
    }
}

struct GrowArgs {
    KvView kv;
    int n;
    const int32_t *row, *n_new;
    int32_t *claim;              // [rows]
    int32_t *first;              // [n] pages wanted by the rows before
    int32_t *have;               // [n] pages the row has
    int32_t *list;               // [n_pages]
};

// As the fork's plan: round trips.  64 rows, 32 tokens each: 10.1 us.
__global__ __launch_bounds__(PL_THREADS) void hx_kv_grow_kernel(GrowArgs a)
{
    __shared__ int64_t s[PL_WAVES];
    const KvView &kv = a.kv;
    claim_rows(a.row, a.n, kv.rows, a.claim);
    bool bad = false;
    int64_t want = 0;
    const int rounds = (a.n + PL_THREADS - 1) / PL_THREADS;
    for (int it = 0; it < rounds; ++it) {
        const int i = it * PL_THREADS + threadIdx.x;
        int need = 0, have = -1;
        if (i < a.n) {
            const int r = a.row[i], m = a.n_new[i];
            if (r >= 0 && r < kv.rows && m >= 0 && hx_sync_load(a.claim + r) == i) {
                const int len = kv.len[r];
                if (hx_row_ok(kv, r, len) && (int64_t)len + m <= (int64_t)kv.max_pages << kv.shift) {
                    have = hx_pages_of(len, kv.shift);
                    need = hx_pages_of(len + m, kv.shift) - have;
                }
            }
            if (have < 0) bad = true;
        }
        int64_t all;
        int64_t before = want + block_before(need, s, &all);
        if (i < a.n) {
            a.first[i] = (int)(before < NO_CLAIM ? before : NO_CLAIM);
            a.have[i] = have;
        }
        want += all;
    }
    if (bad) hx_raise(kv.status, HX_ERR_INDEX);
    const int found = first_pages<false>(kv.ref, 0, kv.n_pages, want < kv.n_pages ? (int)want : kv.n_pages, a.list, s);
    // a page a thread: the row that wanted it is found by bisection
    for (uint32_t j = threadIdx.x; j < (uint32_t)found; j += PL_THREADS) {
        int lo = 0, hi = a.n - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if ((uint32_t)a.first[mid] <= j) lo = mid; else hi = mid - 1;
        }
        // `lo` is the last row before whom at most j pages are wanted: j is its own
        const int r = a.row[lo], need = hx_pages_of(kv.len[r] + a.n_new[lo], kv.shift) - a.have[lo];
        if ((int64_t)a.first[lo] + need > found) continue;       // it does not get all it needs
        const int page = a.list[j];
        kv.ref[page] = 1;
        hx_row(kv, r)[a.have[lo] + (int)j - a.first[lo]] = page;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.n; i += PL_THREADS) {
        if (a.have[i] < 0) continue;
        const int r = a.row[i], len = kv.len[r] + a.n_new[i], need = hx_pages_of(len, kv.shift) - a.have[i];
        if (need > 0 && (int64_t)a.first[i] + need > found) hx_raise(kv.status, HX_ERR_CAPACITY);
        else kv.len[r] = len;
    }
}

// ---- write -------------------------------------------------------------------

__device__ __forceinline__ float load_number(const float *p) { return *p; }
__device__ __forceinline__ float load_number(const __bf16 *p) { return (float)*p; }
__device__ __forceinline__ float load_number(const _Float16 *p) { return (float)*p; }

// 4 numbers as 8 bits each.  The clamp would lose a NaN.
__device__ __forceinline__ uint32_t to_e4m3(const float *x, float scale)
{
    float y[4];
    bool nan[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[i] = x[i] / scale;
        nan[i] = y[i] != y[i];
        y[i] = fminf(fmaxf(y[i], -448.0f), 448.0f);
    }
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (nan[i]) w = (w & ~(0xffu << (8 * i))) | (0x7fu << (8 * i));
    return w;
}

struct WriteArgs {
    KvView kv;
    int layer, n, n_tok;
    const int32_t *row, *tok_ptr;
    const void *k, *v;
    int64_t token_stride, head_stride;
    const float *k_scale, *v_scale;
    bool aligned;            // 8 numbers of a source can be loaded at once
};

// Of a row listed twice the first entry counts.  A wavefront looks for the rows of its lanes' entries among those listed before, 256 at a time
// in registers, the next 256 under way; entries rise with the lanes.
constexpr int LISTED_EACH = 4;
__device__ __forceinline__ void listed_ask(const int32_t *row, int from, int to, int *x)
{
#pragma unroll
    for (int k = 0; k < LISTED_EACH; ++k) {
        const int j = from + k * HX_WAVE + (threadIdx.x & (HX_WAVE - 1));
        x[k] = j < to ? row[j] : 0;
    }
}
// x: the call's first rows; all lanes take part
__device__ __forceinline__ bool listed_before(const int32_t *row, int *x, int entry, int mine)
{
    const int lane = threadIdx.x & (HX_WAVE - 1), most = __builtin_amdgcn_readlane(entry, HX_WAVE - 1);
    bool listed = false;
    for (int j0 = 0; j0 < most; j0 += LISTED_EACH * HX_WAVE) {
        int next[LISTED_EACH];
        listed_ask(row, j0 + LISTED_EACH * HX_WAVE, most, next);
        for (unsigned long long left = ~0ull; left;) {
            const int from = __builtin_ctzll(left), e = __builtin_amdgcn_readlane(entry, from), r = __builtin_amdgcn_readlane(mine, from);
            bool hit = false;
#pragma unroll
            for (int k = 0; k < LISTED_EACH; ++k) hit |= x[k] == r && j0 + k * HX_WAVE + lane < e;
            const bool any = __builtin_amdgcn_ballot_w64(hit) != 0;
            listed |= any && entry == e;
            left &= ~__builtin_amdgcn_ballot_w64(entry == e);
        }
#pragma unroll
        for (int k = 0; k < LISTED_EACH; ++k) x[k] = next[k];
    }
    return listed;
}

// 8 numbers of a key and of a value a thread; D of one byte: e4m3.  2048 tokens of 64 rows, 8 heads of 128 (17 MB read and written):
// 5.2 us in a graph of such calls, most of it the lookups before a thread's store (its sequence by bisection, row, length, page, count).  One
// token each of 256 rows 3.8, of 1024 5.6; of these the look for rows listed twice takes 0.2, 0.3 and 1.1.
template <typename S, typename D>
__global__ __launch_bounds__(CP_THREADS) void hx_kv_write_kernel(WriteArgs a)
{
    const KvView &kv = a.kv;
    const int per_head = kv.dim / 8, per = per_head * kv.n_heads;
    const int64_t u = (int64_t)blockIdx.x * CP_THREADS + threadIdx.x;
    const int64_t q = u / per;
    const int c = (int)(u % per), h = c / per_head, d = (c % per_head) * 8;
    int rows[LISTED_EACH];
    listed_ask(a.row, 0, a.n, rows);
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.tok_ptr[mid] <= q) lo = mid; else hi = mid - 1;
    }
    const int first = a.tok_ptr[lo], last = a.tok_ptr[lo + 1], r = a.row[lo];
    // an entry is written as a whole or not at all
    bool ok = first >= 0 && first <= q && q < last && last <= a.n_tok && r >= 0 && r < kv.rows;
    const int len = ok ? kv.len[r] : 0;
    ok = ok && hx_row_ok(kv, r, len) && last - first <= len;
    const int64_t pos = (int64_t)len - last + q;
    const int page = ok ? hx_row(kv, r)[pos >> kv.shift] : -1;
    ok = page >= 0 && page < kv.n_pages && kv.ref[page] <= 1;
    const bool again = listed_before(a.row, rows, lo, r);
    if (q >= a.n_tok) return;
    if (!ok || again) { if (c == 0) hx_raise(kv.status, HX_ERR_INDEX); return; }
    const int64_t from = q * a.token_stride + h * a.head_stride + d;
    const int64_t to = hx_kv_at(kv, a.layer, page, h, (int)(pos & ((1 << kv.shift) - 1))) + d;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const S *src = (const S *)(which ? a.v : a.k) + from;
        struct alignas(8 * sizeof(S) < 16 ? 8 * sizeof(S) : 16) Eight { S x[8]; } e;
        if (a.aligned) e = *(const Eight *)src;
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) e.x[i] = src[i];
        if constexpr (sizeof(D) == 1) {
            const float *scales = which ? a.v_scale : a.k_scale;
            const float scale = scales ? scales[a.layer * kv.n_heads + h] : 1.0f;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = load_number(&e.x[i]);
            *(uint2 *)((char *)(which ? kv.v : kv.k) + to) = make_uint2(to_e4m3(x, scale), to_e4m3(x + 4, scale));
        } else {
            struct alignas(16) Out { D x[8]; } o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o.x[i] = (D)load_number(&e.x[i]);
            *(Out *)((D *)(which ? kv.v : kv.k) + to) = o;
        }
    }
}

// ---- keep --------------------------------------------------------------------

struct KeepArgs {
    KvView kv;
    int n, n_keep;
    const int32_t *row, *n_draft, *keep_ptr, *keep;
    int32_t *ok;             // [n] whether the row is changed
    int row_bytes;
};

// Whether entry i of the call can be carried out; the same for all threads.  Its answer is taken before anything of the call
// is applied: later the pages' counts may differ.
__device__ bool keep_check(const KeepArgs &a, int i, int *s_bad)
{
    const KvView &kv = a.kv;
    if (threadIdx.x == 0) *s_bad = 0;
    __syncthreads();
    const int r = a.row[i], nd = a.n_draft[i], k0 = a.keep_ptr[i], k1 = a.keep_ptr[i + 1];
    bool bad = r < 0 || r >= kv.rows || nd < 0 || k0 < 0 || k1 < k0 || k1 > a.n_keep;
    const int m = bad ? 0 : k1 - k0;
    bad |= m > nd;
    int len = 0;
    if (!bad) {
        len = kv.len[r];
        bad = !hx_row_ok(kv, r, len) || nd > len;
    }
    if (!bad) {
        const int base = len - nd;
        const int32_t *table = hx_row(kv, r);
        for (int j = threadIdx.x; j < i; j += CP_THREADS) bad |= a.row[j] == r;
        for (uint32_t j = threadIdx.x; j < (uint32_t)m; j += CP_THREADS) {
            const int k = a.keep[k0 + j];
            if (k < 0 || k >= nd || (j > 0 && a.keep[k0 + j - 1] >= k)) { bad = true; continue; }
            if ((uint32_t)k == j) continue;
            const int from = table[(base + k) >> kv.shift], to = table[(base + j) >> kv.shift];
            bad |= from < 0 || from >= kv.n_pages || to < 0 || to >= kv.n_pages || kv.ref[to] > 1;
        }
        // the page that will be filled further must be this row's alone
        if (threadIdx.x == 0 && nd > m && ((base + m) & ((1 << kv.shift) - 1))) {
            const int page = table[(base + m) >> kv.shift];
            bad |= page >= kv.n_pages || (page >= 0 && kv.ref[page] > 1);
        }
    }
    if (bad) *s_bad = 1;
    __syncthreads();
    return !*s_bad;
}

// 64 rows, up to 6 of 32 tokens kept, one layer: 7.3 us, 3.1 more for the tables; moves of a row follow each other.  With the tables, 32 layers
// of 64, 256 and 1024 rows: 18, 55 and 318 us, for 49, 193 and 785 MB read and written (each layer's workgroups check their row again).
// Workgroup (i, 2 layer + v): a token's place is read by the thread that then writes the earlier place, and numbers rise, so what
// a thread overwrites it has read.
__global__ __launch_bounds__(CP_THREADS) void hx_kv_keep_move_kernel(KeepArgs a)
{
    __shared__ int s_bad;
    const KvView &kv = a.kv;
    const int parts = 2 * kv.n_layers, i = blockIdx.x / parts, part = blockIdx.x % parts;
    const bool ok = keep_check(a, i, &s_bad);
    if (part == 0 && threadIdx.x == 0) {
        a.ok[i] = ok;
        if (!ok) hx_raise(kv.status, HX_ERR_INDEX);
    }
    if (!ok) return;
    const int r = a.row[i], k0 = a.keep_ptr[i], m = a.keep_ptr[i + 1] - k0, base = kv.len[r] - a.n_draft[i];
    const int32_t *table = hx_row(kv, r);
    char *store = (char *)((part & 1) ? kv.v : kv.k);
    const int64_t head_bytes = (int64_t)a.row_bytes << kv.shift;
    const int64_t layer_page = (int64_t)(part >> 1) * kv.n_pages;
    const int per_head = a.row_bytes / 16, in_page = (1 << kv.shift) - 1;
    for (int c = threadIdx.x; c < per_head * kv.n_heads; c += CP_THREADS) {
        char *at = store + (c / per_head) * head_bytes + (c % per_head) * 16;
        for (int j = 0; j < m; ++j) {
            const int k = a.keep[k0 + j];
            if (k == j) continue;
            const int from = base + k, to = base + j;
            const char *x = at + (layer_page + table[from >> kv.shift]) * kv.n_heads * head_bytes + (int64_t)(from & in_page) * a.row_bytes;
            char *y = at + (layer_page + table[to >> kv.shift]) * kv.n_heads * head_bytes + (int64_t)(to & in_page) * a.row_bytes;
            *(uint4 *)y = *(const uint4 *)x;
        }
    }
}

// A page is held by one table less.  Counts that would go below 0 stay.
__device__ __forceinline__ void give_back(const KvView &kv, int page)
{
    if (page >= kv.n_pages) { hx_raise(kv.status, HX_ERR_INDEX); return; }
    if (atomicSub(kv.ref + page, 1) <= 0) { atomicAdd(kv.ref + page, 1); hx_raise(kv.status, HX_ERR_INDEX); }
}

__global__ __launch_bounds__(CP_THREADS) void hx_kv_keep_apply_kernel(KeepArgs a)
{
    const KvView &kv = a.kv;
    const int i = blockIdx.x;
    if (!a.ok[i]) return;
    const int r = a.row[i], len = kv.len[r], left = len - a.n_draft[i] + a.keep_ptr[i + 1] - a.keep_ptr[i];
    int32_t *table = hx_row(kv, r);
    for (uint32_t b = hx_pages_of(left, kv.shift) + threadIdx.x; b < (uint32_t)hx_pages_of(len, kv.shift); b += CP_THREADS) {
        const int page = table[b];
        table[b] = -1;
        if (page >= 0) give_back(kv, page);
    }
    __syncthreads();
    if (threadIdx.x == 0) kv.len[r] = left;
}

// ---- free --------------------------------------------------------------------

struct FreeArgs {
    KvView kv;
    int n;
    const int32_t *row, *first, *last;
};

// 2 us for a row, 4 to 5 for 24 or 64.
// A workgroup a row.  An entry is taken out by an exchange, so a row that is listed twice gives each page back once.
__global__ __launch_bounds__(CP_THREADS) void hx_kv_free_kernel(FreeArgs a)
{
    const KvView &kv = a.kv;
    const int i = blockIdx.x, r = a.row[i];
    if (r < 0 || r >= kv.rows) { if (threadIdx.x == 0) hx_raise(kv.status, HX_ERR_INDEX); return; }
    const int len = hx_sync_load(kv.len + r);
    if (!hx_row_ok(kv, r, len)) { if (threadIdx.x == 0) hx_raise(kv.status, HX_ERR_INDEX); return; }
    const HxSpan span = a.first ? hx_filled_within(a.first[i], a.last[i], len, kv.shift) : HxSpan{0, (uint32_t)hx_pages_of(len, kv.shift)};
    int32_t *table = hx_row(kv, r);
    for (uint32_t b = span.lo + threadIdx.x; b < span.hi; b += CP_THREADS) {
        const int page = atomicExch(table + b, -1);
        if (page >= 0) give_back(kv, page);
    }
    if (a.first) return;
    __syncthreads();
    if (threadIdx.x == 0) __hip_atomic_store(kv.len + r, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---- compact -----------------------------------------------------------------

struct CompactArgs {
    KvView kv;
    int32_t *count;              // pages that move
    int32_t *high, *hole;        // [n_pages / 2] which, and where to
    int32_t *moved;              // [n_pages]
    int32_t *n_used;             // or NULL
    int64_t page_bytes;          // of a page in one layer's keys
};

// Three launches: which pages move (9 us for 3882 pages), the copy, the tables (4.4 us).  The copy is bound by HBM: 3.8 GB read and written in
// 776 us, 4.9 TB/s, a plain copy's rate.
__global__ __launch_bounds__(PL_THREADS) void hx_kv_compact_plan_kernel(CompactArgs a)
{
    __shared__ int64_t s[PL_WAVES];
    const KvView &kv = a.kv;
    int mine = 0;
    for (uint32_t p = threadIdx.x; p < (uint32_t)kv.n_pages; p += PL_THREADS) {
        const bool used = kv.ref[p] > 0;
        mine += used;
        a.moved[p] = used ? (int)p : -1;
    }
    int64_t all;
    (void)block_before(mine, s, &all);
    const int used = (int)all;
    const int n = first_pages<true>(kv.ref, used, kv.n_pages, kv.n_pages, a.high, s);
    first_pages<false>(kv.ref, 0, used, n, a.hole, s);
    for (int j = threadIdx.x; j < n; j += PL_THREADS) a.moved[a.high[j]] = a.hole[j];
    if (threadIdx.x == 0) {
        *a.count = n;
        if (a.n_used) *a.n_used = used;
    }
}

__global__ __launch_bounds__(CP_THREADS) void hx_kv_compact_copy_kernel(CompactArgs a)
{
    const KvView &kv = a.kv;
    const int n = *a.count, parts = 2 * kv.n_layers;
    for (int64_t u = blockIdx.x; u < (int64_t)n * parts; u += gridDim.x) {
        const int j = (int)(u / parts), part = (int)(u % parts);
        char *store = (char *)((part & 1) ? kv.v : kv.k) + (int64_t)(part >> 1) * kv.n_pages * a.page_bytes;
        const uint4 *from = (const uint4 *)(store + a.high[j] * a.page_bytes);
        uint4 *to = (uint4 *)(store + a.hole[j] * a.page_bytes);
        for (int64_t c = threadIdx.x; c < a.page_bytes / 16; c += CP_THREADS) to[c] = from[c];
    }
}

__global__ __launch_bounds__(CP_THREADS) void hx_kv_compact_apply_kernel(CompactArgs a)
{
    const KvView &kv = a.kv;
    const int64_t first = (int64_t)blockIdx.x * CP_THREADS + threadIdx.x, step = (int64_t)gridDim.x * CP_THREADS;
    for (int64_t i = first; i < (int64_t)kv.rows * kv.max_pages; i += step) {
        const int page = kv.table[i];
        if (page < 0) continue;
        if (page >= kv.n_pages) { hx_raise(kv.status, HX_ERR_INDEX); continue; }
        kv.table[i] = a.moved[page];
    }
    for (int64_t j = first; j < *a.count; j += step) {
        kv.ref[a.hole[j]] = kv.ref[a.high[j]];
        kv.ref[a.high[j]] = 0;
    }
}

int blocks_for(int64_t items, int threads, int64_t most)
{
    const int64_t b = (items + threads - 1) / threads;
    return (int)(b < 1 ? 1 : b > most ? most : b);
}

}  // namespace

#define HX_KV_BEGIN(ctx, what_ok, groups)                                                           \
    KvView kv;                                                                                      \
    if (int rc_ = hx_kv_view(ctx, pool, seqs, &kv)) return rc_;                                     \
    HX_REQUIRE(ctx, n >= 0, HX_ERR_INVALID_ARG, "negative size");                                   \
    if (n == 0) return HX_OK;                                                                       \
    HX_REQUIRE(ctx, what_ok, HX_ERR_INVALID_ARG, "NULL array");                                     \
    HX_REQUIRE(ctx, kv.rows > 0, HX_ERR_INVALID_ARG, "%d rows asked for of no sequences", n);       \
    HX_REQUIRE(ctx, (int64_t)n * (groups) <= hx_most_groups(CP_THREADS), HX_ERR_SHAPE, "%d rows of %d layers in one call", n, kv.n_layers); \
    hipStream_t stream = (hipStream_t)stream_

#define HX_KV_DEVICE(ctx)                                                                           \
    HxDeviceGuard guard(ctx->device);                                                               \
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device)

extern "C" int hx_kv_fork(hx_ctx *ctx, const hx_kv_pool *pool, const hx_kv_seqs *seqs, int32_t n,
                          const int32_t *src, const int32_t *dst, const int32_t *n_tok, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    HX_KV_BEGIN(ctx, src && dst, 1 + 2 * kv.n_layers);
    const int parts = 1 + 2 * kv.n_layers;
    HX_KV_DEVICE(ctx);
    if (int rc = hx_scratch(ctx, hx_serve(ctx)->kv, ((size_t)kv.rows + 4 * (size_t)n) * sizeof(int32_t), stream)) return rc;
    int32_t *w = (int32_t *)hx_serve(ctx)->kv.p;
    ForkArgs a{kv, n, src, dst, n_tok, w, w + kv.rows, w + kv.rows + n, w + kv.rows + 2 * (size_t)n, w + kv.rows + 3 * (size_t)n,
               pool->head_dim * hx_type_size(pool->dtype)};
    hx_kv_fork_plan_kernel<<<1, PL_THREADS, 0, stream>>>(a);
    hx_kv_fork_copy_kernel<<<n * parts, CP_THREADS, 0, stream>>>(a);
    return hx_check_launch(ctx, "hx_kv_fork_copy_kernel");
}

extern "C" int hx_kv_grow(hx_ctx *ctx, const hx_kv_pool *pool, const hx_kv_seqs *seqs, int32_t n,
                          const int32_t *row, const int32_t *n_new, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    HX_KV_BEGIN(ctx, row && n_new, 1);
    HX_KV_DEVICE(ctx);
    if (int rc = hx_scratch(ctx, hx_serve(ctx)->kv, ((size_t)kv.rows + 2 * (size_t)n + kv.n_pages) * sizeof(int32_t), stream)) return rc;
    int32_t *w = (int32_t *)hx_serve(ctx)->kv.p;
    GrowArgs a{kv, n, row, n_new, w, w + kv.rows, w + kv.rows + n, w + kv.rows + 2 * (size_t)n};
    hx_kv_grow_kernel<<<1, PL_THREADS, 0, stream>>>(a);
    return hx_check_launch(ctx, "hx_kv_grow_kernel");
}

extern "C" int hx_kv_write(hx_ctx *ctx, const hx_kv_pool *pool, int32_t layer, const hx_kv_seqs *seqs, int32_t n,
                           const int32_t *row, const int32_t *tok_ptr, int32_t n_tok, int32_t src_dtype,
                           const void *k, const void *v, int64_t token_stride, int64_t head_stride, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    HX_KV_BEGIN(ctx, row && tok_ptr, 1);
    HX_REQUIRE(ctx, layer >= 0 && layer < kv.n_layers, HX_ERR_INVALID_ARG, "layer %d of %d", layer, kv.n_layers);
    HX_REQUIRE(ctx, n_tok >= 0, HX_ERR_INVALID_ARG, "negative size");
    HX_REQUIRE(ctx, src_dtype == HX_F32 || src_dtype == HX_BF16 || src_dtype == HX_F16, HX_ERR_INVALID_ARG, "source of type %d", src_dtype);
    if (n_tok == 0) return HX_OK;
    HX_REQUIRE(ctx, k && v, HX_ERR_INVALID_ARG, "NULL keys or values");
    HX_REQUIRE(ctx, (((uintptr_t)k | (uintptr_t)v) & (hx_type_size(src_dtype) - 1)) == 0, HX_ERR_INVALID_ARG, "keys or values are not aligned to their type");
    const bool aligned = (((uintptr_t)k | (uintptr_t)v) & 15) == 0 && token_stride % 8 == 0 && head_stride % 8 == 0;
    WriteArgs a{kv, layer, n, n_tok, row, tok_ptr, k, v, token_stride, head_stride, pool->k_scale, pool->v_scale, aligned};
    const int64_t blocks = ((int64_t)n_tok * (kv.dim / 8) * kv.n_heads + CP_THREADS - 1) / CP_THREADS;
    HX_REQUIRE(ctx, blocks <= hx_most_groups(CP_THREADS), HX_ERR_SHAPE, "%d tokens in one call", n_tok);
    const int grid = (int)blocks;
    HX_KV_DEVICE(ctx);
#define HX_WRITE(S)                                                                                              \
    (pool->dtype == HX_BF16 ? hx_kv_write_kernel<S, __bf16><<<grid, CP_THREADS, 0, stream>>>(a)                  \
     : pool->dtype == HX_F16 ? hx_kv_write_kernel<S, _Float16><<<grid, CP_THREADS, 0, stream>>>(a)               \
                             : hx_kv_write_kernel<S, uint8_t><<<grid, CP_THREADS, 0, stream>>>(a))
    if (src_dtype == HX_F32) HX_WRITE(float);
    else if (src_dtype == HX_BF16) HX_WRITE(__bf16);
    else HX_WRITE(_Float16);
#undef HX_WRITE
    return hx_check_launch(ctx, "hx_kv_write_kernel");
}

extern "C" int hx_kv_keep(hx_ctx *ctx, const hx_kv_pool *pool, const hx_kv_seqs *seqs, int32_t n, const int32_t *row,
                          const int32_t *n_draft, const int32_t *keep_ptr, const int32_t *keep, int32_t n_keep, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    HX_KV_BEGIN(ctx, row && n_draft && keep_ptr, 2 * kv.n_layers);
    HX_REQUIRE(ctx, n_keep >= 0, HX_ERR_INVALID_ARG, "negative size");
    HX_REQUIRE(ctx, n_keep == 0 || keep, HX_ERR_INVALID_ARG, "NULL array");
    const int parts = 2 * kv.n_layers;
    HX_KV_DEVICE(ctx);
    if (int rc = hx_scratch(ctx, hx_serve(ctx)->kv, (size_t)n * sizeof(int32_t), stream)) return rc;
    KeepArgs a{kv, n, n_keep, row, n_draft, keep_ptr, keep, (int32_t *)hx_serve(ctx)->kv.p, pool->head_dim * hx_type_size(pool->dtype)};
    hx_kv_keep_move_kernel<<<n * parts, CP_THREADS, 0, stream>>>(a);
    hx_kv_keep_apply_kernel<<<n, CP_THREADS, 0, stream>>>(a);
    return hx_check_launch(ctx, "hx_kv_keep_apply_kernel");
}

extern "C" int hx_kv_free(hx_ctx *ctx, const hx_kv_pool *pool, const hx_kv_seqs *seqs, int32_t n, const int32_t *row,
                          const int32_t *first, const int32_t *last, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    HX_KV_BEGIN(ctx, row, 1);
    HX_REQUIRE(ctx, !first == !last, HX_ERR_INVALID_ARG, "first and last go together");
    HX_KV_DEVICE(ctx);
    FreeArgs a{kv, n, row, first, last};
    hx_kv_free_kernel<<<n, CP_THREADS, 0, stream>>>(a);
    return hx_check_launch(ctx, "hx_kv_free_kernel");
}

extern "C" int hx_kv_compact(hx_ctx *ctx, const hx_kv_pool *pool, const hx_kv_seqs *seqs, int32_t *n_used, int32_t *moved, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    KvView kv;
    if (int rc = hx_kv_view(ctx, pool, seqs, &kv)) return rc;
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    hipStream_t stream = (hipStream_t)stream_;
    const size_t P = kv.n_pages;
    if (int rc = hx_scratch(ctx, hx_serve(ctx)->kv, (4 + 3 * P) * sizeof(int32_t), stream)) return rc;
    int32_t *w = (int32_t *)hx_serve(ctx)->kv.p;
    const int64_t page_bytes = ((int64_t)kv.n_heads << kv.shift) * kv.dim * hx_type_size(pool->dtype);
    CompactArgs a{kv, w, w + 4, w + 4 + P, moved ? moved : w + 4 + 2 * P, n_used, page_bytes};
    hx_kv_compact_plan_kernel<<<1, PL_THREADS, 0, stream>>>(a);
    if (P > 0) {
        // how many pages move only the GPU knows: at most half of them
        const int64_t most = (int64_t)(P / 2 + 1) * 2 * kv.n_layers;
        hx_kv_compact_copy_kernel<<<(int)(most < 16 * ctx->num_cu ? most : 16 * ctx->num_cu), CP_THREADS, 0, stream>>>(a);
        const int64_t entries = (int64_t)kv.rows * kv.max_pages;
        hx_kv_compact_apply_kernel<<<blocks_for(entries > (int64_t)P ? entries : P, CP_THREADS, 8 * ctx->num_cu), CP_THREADS, 0, stream>>>(a);
    }
    return hx_check_launch(ctx, "hx_kv_compact_apply_kernel");
}
