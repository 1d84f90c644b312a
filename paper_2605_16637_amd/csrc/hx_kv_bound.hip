// Bounds of keys: the least and the largest number of a page's keys in every place.
#include "hx_kv_numbers.hpp"

namespace {

constexpr int BD_THREADS = 256;

struct BoundArgs {
    KvView kv;
    int layer, layers, n, each;        // layers: how many, from `layer` on; each: workgroups of a row's layer
    const int32_t *row, *n_new;
    const uint8_t *k_exp;
    void *bounds;
};

// 16 bytes of a token's key a thread, token after token of a page; a wavefront's threads lie beside each other in a head, then in the next.
// A workgroup takes every `each`-th of a row's threads-full of pages.  Bound by the keys' bytes: 16 prompts of some 4000 tokens, 8 heads of 128, pages of 16:
// 160 MB read, 20 written in 50 us, 3.6 TB/s (over the same keys again and again, part of which the 256 MB cache then holds, 40).  The pages of the last
// tokens of 64 rows: 5 to 8 us in one layer, lookups and a page's tokens one after the other, 10 to 14 in 32.
template <typename S, typename B>
__global__ __launch_bounds__(BD_THREADS) void hx_kv_bound_kernel(BoundArgs a)
{
    constexpr int N = std::is_same_v<S, E2m1> ? 32 : 16 / (int)sizeof(S);
    const KvView &kv = a.kv;
    const int i = blockIdx.x % a.n, rest = blockIdx.x / a.n, layer = a.layer + rest % a.layers, part = rest / a.layers, r = a.row[i];
    const bool first = rest == 0 && threadIdx.x == 0;
    if (r < 0 || r >= kv.rows) { if (first) hx_raise(kv.status, HX_ERR_INDEX); return; }
    const int len = kv.len[r], fresh = a.n_new ? a.n_new[i] : len;
    if (!hx_row_ok(kv, r, len) || fresh < 0 || fresh > len) { if (first) hx_raise(kv.status, HX_ERR_INDEX); return; }
    if (fresh == 0) return;
    const int b0 = (len - fresh) >> kv.shift, b1 = hx_pages_of(len, kv.shift), T = 1 << kv.shift;
    const int per_head = kv.dim / N, per = per_head * kv.n_heads;
    const int32_t *table = hx_row(kv, r);
    for (int64_t u = (int64_t)part * BD_THREADS + threadIdx.x; u < (int64_t)(b1 - b0) * per; u += (int64_t)a.each * BD_THREADS) {
        const int b = b0 + (int)(u / per), c = (int)(u % per), head = c / per_head, d = c % per_head * N, page = table[b];
        if (page < 0) continue;
        if (page >= kv.n_pages) { hx_raise(kv.status, HX_ERR_INDEX); continue; }
        const int64_t left = (int64_t)len - ((int64_t)b << kv.shift);
        const int filled = left < T ? (int)left : T;
        float lo[N], hi[N];
#pragma unroll
        for (int j = 0; j < N; ++j) { lo[j] = __builtin_inff(); hi[j] = -__builtin_inff(); }
        const int64_t at = hx_kv_at(kv, layer, page, head, 0) + d;
#pragma unroll 4
        for (int t = 0; t < filled; ++t) {
            float x[N];
            stored<S, N>(kv.k, a.k_exp, 1.0f, at + (int64_t)t * kv.dim, x);
#pragma unroll
            for (int j = 0; j < N; ++j) { lo[j] = fminf(lo[j], x[j]); hi[j] = fmaxf(hi[j], x[j]); }
        }
        struct alignas(16) Out { B x[N]; } o;
        B *to = (B *)a.bounds + (((int64_t)layer * kv.n_pages + page) * kv.n_heads + head) * 2 * kv.dim + d;
#pragma unroll
        for (int j = 0; j < N; ++j) o.x[j] = (B)lo[j];
        *(Out *)to = o;
#pragma unroll
        for (int j = 0; j < N; ++j) o.x[j] = (B)hi[j];
        *(Out *)(to + kv.dim) = o;
    }
}

}  // namespace

extern "C" int hx_kv_bound(hx_ctx *ctx, const hx_kv_pool *pool, int32_t layer, const hx_kv_seqs *seqs, int32_t n,
                           const int32_t *row, const int32_t *n_new, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    KvView kv;
    if (int rc = hx_kv_view(ctx, pool, seqs, &kv)) return rc;
    HX_REQUIRE(ctx, n >= 0, HX_ERR_INVALID_ARG, "negative size");
    HX_REQUIRE(ctx, layer >= -1 && layer < kv.n_layers, HX_ERR_INVALID_ARG, "layer %d of %d", layer, kv.n_layers);
    HX_REQUIRE(ctx, pool->bounds || kv.n_pages == 0, HX_ERR_INVALID_ARG, "a pool without bounds");
    if (n == 0 || kv.n_pages == 0) return HX_OK;
    HX_REQUIRE(ctx, row, HX_ERR_INVALID_ARG, "NULL array");
    HX_REQUIRE(ctx, kv.rows > 0, HX_ERR_INVALID_ARG, "%d rows asked for of no sequences", n);
    const int layers = layer < 0 ? kv.n_layers : 1;
    // how many pages a row has only the GPU knows: workgroups for all that its entries could be, up to some 32 a CU in all, and one a row at least
    const int N = pool->dtype == HX_E2M1 ? 32 : pool->dtype == HX_E4M3 ? 16 : 8;
    const int64_t could = ((int64_t)kv.max_pages * kv.n_heads * (kv.dim / N) + BD_THREADS - 1) / BD_THREADS, few = 32 * (int64_t)ctx->num_cu / ((int64_t)n * layers);
    const int64_t part = could < few ? could : few, each = part > 1 ? part : 1, grid = each * n * layers;
    HX_REQUIRE(ctx, grid <= hx_most_groups(BD_THREADS), HX_ERR_SHAPE, "%d rows of %d layers in one call", n, layers);
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    const hipStream_t stream = (hipStream_t)stream_;
    const BoundArgs a{kv, layer < 0 ? 0 : layer, layers, n, (int)each, row, n_new, pool->k_exp, pool->bounds};
    if (pool->dtype == HX_BF16) hx_kv_bound_kernel<__bf16, __bf16><<<(int)grid, BD_THREADS, 0, stream>>>(a);
    else if (pool->dtype == HX_F16) hx_kv_bound_kernel<_Float16, _Float16><<<(int)grid, BD_THREADS, 0, stream>>>(a);
    else if (pool->dtype == HX_E4M3) hx_kv_bound_kernel<uint8_t, __bf16><<<(int)grid, BD_THREADS, 0, stream>>>(a);
    else hx_kv_bound_kernel<E2m1, __bf16><<<(int)grid, BD_THREADS, 0, stream>>>(a);
    return hx_check_launch(ctx, "hx_kv_bound_kernel");
}
