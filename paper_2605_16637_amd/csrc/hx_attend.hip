// Attention over cached pages: the entry point.  The kernels are hx_attend.hpp's, compiled for a pair of types in each of hx_attend_*.hip.
#include "hx_attend_args.hpp"

#include <cmath>

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
    HX_REQUIRE(ctx, std::isfinite(g.scale), HX_ERR_INVALID_ARG, "scale is not finite");
    if (g.n == 0 || g.n_q == 0 || g.max_q == 0) return HX_OK;
    HX_REQUIRE(ctx, g.q_ptr && g.q && g.out, HX_ERR_INVALID_ARG, "NULL array");
    HX_REQUIRE(ctx, (((uintptr_t)g.q | (uintptr_t)g.out) & 1) == 0, HX_ERR_INVALID_ARG, "q or out is not aligned to its type");
    HX_REQUIRE(ctx, kv.rows > 0, HX_ERR_INVALID_ARG, "%d sequences asked for of none", g.n);
    HX_REQUIRE(ctx, (int64_t)g.max_q * g.n_heads <= INT32_MAX / 2 && (int64_t)g.n * kv.n_heads <= INT32_MAX, HX_ERR_SHAPE,
               "%d queries of %d heads, %d sequences", g.max_q, g.n_heads, g.n);
    HX_REQUIRE(ctx, (int64_t)kv.max_pages << kv.shift <= INT32_MAX / 2, HX_ERR_SHAPE, "%d pages of %d tokens a row", kv.max_pages, 1 << kv.shift);
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    hipStream_t stream = (hipStream_t)stream_;
    HxAttend a{};
    a.kv = kv;
    a.layer = layer; a.n = g.n; a.row = g.row; a.q_ptr = g.q_ptr; a.n_q = g.n_q;
    a.max_q = g.max_q < g.n_q ? g.max_q : g.n_q;
    a.n_heads = g.n_heads; a.group = g.n_heads / kv.n_heads;
    a.q = g.q; a.q_token = g.q_token; a.q_head = g.q_head;
    a.out = g.out; a.out_token = g.out_token; a.out_head = g.out_head;
    a.lse = g.lse; a.scale = g.scale; a.window = g.window; a.n_sink = g.n_sink; a.parent = g.parent;
    a.zeros = hx_serve(ctx)->d_zeros;
    a.k_scale = pool->k_scale; a.v_scale = pool->v_scale;
    a.q_wide = ((uintptr_t)g.q & 15) == 0 && g.q_token % 8 == 0 && g.q_head % 8 == 0;
    a.out_wide = ((uintptr_t)g.out & 7) == 0 && g.out_token % 4 == 0 && g.out_head % 4 == 0;
    const bool fp8 = pool->dtype == HX_E4M3;
    if (g.dtype == HX_BF16) return fp8 ? hx_attend_bf16_e4m3(ctx, a, g.max_len, stream) : hx_attend_bf16(ctx, a, g.max_len, stream);
    return fp8 ? hx_attend_f16_e4m3(ctx, a, g.max_len, stream) : hx_attend_f16(ctx, a, g.max_len, stream);
}
