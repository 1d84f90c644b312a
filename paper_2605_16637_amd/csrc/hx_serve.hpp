// What the serving step's files share: its part of a context, the cache's addresses, its number types, and checks of its descriptors.
#pragma once

#include "hx_common.hpp"
#include "hx_kv_span.hpp"

// Scratch that grows and never shrinks.  What it was before stays allocated until the context ends: a captured graph may still use
// it, and the sizes double, so all of it together is at most as much again.
struct HxScratch {
    void *p = nullptr;
    size_t cap = 0;
    void *old[48] = {};
    int n_old = 0;
};

// Every context is one of these; the planner's files, which do without, know its first part alone.
struct HxServe : hx_ctx {
    HxScratch kv, att, att_done;           // pages (hx_kv.hip), attention (hx_attend.hip), and its counters, which are 0 between launches
    unsigned att_allowed = 0;              // pairs of types and head_dims whose kernels have been allowed their LDS (hx_attend.hpp)
    int32_t *d_zeros = nullptr;            // 64 words that stay 0
};
inline HxServe *hx_serve(hx_ctx *ctx) { return static_cast<HxServe *>(ctx); }

// Workgroups of `threads` that a launch may have: the runtime counts threads in 32 bits.
constexpr int64_t hx_most_groups(int threads) { return UINT32_MAX / threads; }

inline int hx_scratch(hx_ctx *ctx, HxScratch &s, size_t bytes, hipStream_t stream)
{
    if (bytes <= s.cap) return HX_OK;
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    HX_HIP(ctx, hipStreamIsCapturing(stream, &capture));
    HX_REQUIRE(ctx, capture == hipStreamCaptureStatusNone, HX_ERR_CAPACITY, "scratch would grow by a call that is being captured: make the call once before");
    size_t want = 2 * s.cap > ((size_t)1 << 20) ? 2 * s.cap : (size_t)1 << 20;
    want = bytes > want ? bytes : want;
    HX_REQUIRE(ctx, s.n_old < 48, HX_ERR_CAPACITY, "scratch has grown too often");
    void *p = nullptr;
    const hipError_t e = hipMalloc(&p, want);
    if (e != hipSuccess) {
        (void)hipGetLastError();                   // not the next launch's
        return hx_fail(ctx, HX_ERR_DEVICE, "%zu bytes of scratch: %s", want, hipGetErrorString(e));
    }
    if (s.p) s.old[s.n_old++] = s.p;
    s.p = p;
    s.cap = want;
    return HX_OK;
}

inline void hx_scratch_release(HxScratch &s)
{
    if (s.p) (void)hipFree(s.p);
    for (int i = 0; i < s.n_old; ++i) (void)hipFree(s.old[i]);
    s = HxScratch{};
}

// The pool and the tables as kernels take them.  T = 1 << shift tokens a page.
struct KvView {
    void *k, *v;
    int32_t *ref;
    int32_t *table, *len;
    int32_t *status;
    int n_layers, n_pages, n_heads, shift, dim;
    int rows, max_pages;
};

inline int hx_type_size(int dtype) { return dtype == HX_F32 ? 4 : dtype == HX_E4M3 ? 1 : 2; }

// Fills a view after the checks every call makes.
inline int hx_kv_view(hx_ctx *ctx, const hx_kv_pool *pool, const hx_kv_seqs *seqs, KvView *out)
{
    HX_REQUIRE(ctx, pool && seqs, HX_ERR_INVALID_ARG, "NULL pool or sequences");
    HX_REQUIRE(ctx, pool->n_layers > 0 && pool->n_pages >= 0 && pool->n_heads > 0 && pool->head_dim > 0, HX_ERR_INVALID_ARG,
               "pool of %d layers, %d pages, %d heads of %d", pool->n_layers, pool->n_pages, pool->n_heads, pool->head_dim);
    HX_REQUIRE(ctx, pool->dtype == HX_BF16 || pool->dtype == HX_F16 || pool->dtype == HX_E4M3, HX_ERR_INVALID_ARG, "pool of type %d", pool->dtype);
    const int T = pool->page_tokens;
    HX_REQUIRE(ctx, T >= 1 && T <= HX_MAX_PAGE_TOKENS && (T & (T - 1)) == 0, HX_ERR_SHAPE,
               "page_tokens %d is no power of two up to %d", T, HX_MAX_PAGE_TOKENS);
    HX_REQUIRE(ctx, pool->head_dim % 16 == 0 && pool->head_dim <= 1024, HX_ERR_SHAPE, "head_dim %d is no multiple of 16 up to 1024", pool->head_dim);
    HX_REQUIRE(ctx, pool->n_heads <= 65536 && pool->n_layers <= 65536, HX_ERR_SHAPE, "%d layers of %d heads", pool->n_layers, pool->n_heads);
    HX_REQUIRE(ctx, (int64_t)pool->n_heads * T * pool->head_dim * hx_type_size(pool->dtype) <= INT32_MAX, HX_ERR_SHAPE,
               "a page of %d heads, %d tokens and %d numbers is beyond int32", pool->n_heads, T, pool->head_dim);
    HX_REQUIRE(ctx, pool->n_pages == 0 || (pool->k && pool->v && pool->ref), HX_ERR_INVALID_ARG, "NULL member in pool");
    HX_REQUIRE(ctx, (((uintptr_t)pool->k | (uintptr_t)pool->v) & 15) == 0, HX_ERR_INVALID_ARG, "the pool's k and v have to be 16-byte aligned");
    HX_REQUIRE(ctx, pool->dtype == HX_E4M3 || (!pool->k_scale && !pool->v_scale), HX_ERR_INVALID_ARG, "scales are for a pool of HX_E4M3");
    HX_REQUIRE(ctx, seqs->n >= 0 && seqs->max_pages >= 0, HX_ERR_INVALID_ARG, "negative size of sequences");
    HX_REQUIRE(ctx, (int64_t)seqs->max_pages * T <= INT32_MAX, HX_ERR_SHAPE, "%d pages of %d tokens a row are beyond int32", seqs->max_pages, T);
    HX_REQUIRE(ctx, seqs->n == 0 || (seqs->len && (seqs->table || seqs->max_pages == 0)), HX_ERR_INVALID_ARG, "NULL member in sequences");
    int shift = 0;
    while ((1 << shift) < T) ++shift;
    *out = KvView{pool->k, pool->v, pool->ref, seqs->table, seqs->len, ctx->d_status, pool->n_layers, pool->n_pages, pool->n_heads, shift,
                  pool->head_dim, seqs->n, seqs->max_pages};
    return HX_OK;
}

// a row of the tables whose length its entries can hold
__device__ __forceinline__ bool hx_row_ok(const KvView &kv, int r, int len) { return len >= 0 && len <= (int64_t)kv.max_pages << kv.shift; }

__device__ __forceinline__ int32_t *hx_row(const KvView &kv, int r) { return kv.table + (int64_t)r * kv.max_pages; }

// numbers before (page, head, token) of a layer
__device__ __forceinline__ int64_t hx_kv_at(const KvView &kv, int layer, int page, int head, int tok)
{
    return ((((int64_t)layer * kv.n_pages + page) * kv.n_heads + head) << kv.shift) * kv.dim + (int64_t)tok * kv.dim;
}

__device__ __forceinline__ int hx_sync_load(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
