// Attention over cached pages: the entry point, and the checks that others of its arguments share.  The kernels are hx_attend.hpp's, compiled for a
// pair of types in each of hx_attend_*.hip.
#include "hx_attend_args.hpp"

#include <cmath>

int hx_attend_check(hx_ctx *ctx, const hx_kv_pool *pool, int layer, const KvView &kv, const hx_attend_args *args, bool with_out, bool *any)
{
    *any = false;
    HX_REQUIRE(ctx, args, HX_ERR_INVALID_ARG, "NULL arguments");
    const hx_attend_args &g = *args;
    HX_REQUIRE(ctx, layer >= 0 && layer < kv.n_layers, HX_ERR_INVALID_ARG, "layer %d of %d", layer, kv.n_layers);
    HX_REQUIRE(ctx, kv.dim == 64 || kv.dim == 128 || kv.dim == 256, HX_ERR_SHAPE, "head_dim %d is none of 64, 128, 256", kv.dim);
    HX_REQUIRE(ctx, g.n >= 0 && g.n_q >= 0 && g.max_q >= 0 && g.max_len >= 0 && g.window >= 0 && g.n_sink >= 0, HX_ERR_INVALID_ARG, "negative size");
    HX_REQUIRE(ctx, g.dtype == HX_BF16 || g.dtype == HX_F16, HX_ERR_INVALID_ARG, "queries of type %d", g.dtype);
    HX_REQUIRE(ctx, pool->dtype == HX_E4M3 || pool->dtype == HX_E2M1 || pool->dtype == g.dtype, HX_ERR_INVALID_ARG, "queries of type %d over a pool of type %d", g.dtype, pool->dtype);
    HX_REQUIRE(ctx, g.n_heads > 0 && g.n_heads % kv.n_heads == 0, HX_ERR_SHAPE, "%d query heads over %d KV heads", g.n_heads, kv.n_heads);
    HX_REQUIRE(ctx, !g.parent || g.max_q <= HX_MAX_DRAFTS, HX_ERR_SHAPE, "a tree of up to %d drafts, beyond %d", g.max_q, HX_MAX_DRAFTS);
    HX_REQUIRE(ctx, std::isfinite(g.scale), HX_ERR_INVALID_ARG, "scale is not finite");
    if (g.n == 0 || g.n_q == 0 || g.max_q == 0) return HX_OK;
    HX_REQUIRE(ctx, g.q_ptr && g.q && (g.out || !with_out), HX_ERR_INVALID_ARG, "NULL array");
    HX_REQUIRE(ctx, (((uintptr_t)g.q | (with_out ? (uintptr_t)g.out : 0)) & 1) == 0, HX_ERR_INVALID_ARG, "q or out is not aligned to its type");
    HX_REQUIRE(ctx, kv.rows > 0, HX_ERR_INVALID_ARG, "%d sequences asked for of none", g.n);
    HX_REQUIRE(ctx, (int64_t)g.max_q * g.n_heads <= INT32_MAX / 2 && (int64_t)g.n * kv.n_heads <= INT32_MAX, HX_ERR_SHAPE,
               "%d queries of %d heads, %d sequences", g.max_q, g.n_heads, g.n);
    HX_REQUIRE(ctx, (int64_t)kv.max_pages << kv.shift <= INT32_MAX / 2, HX_ERR_SHAPE, "%d pages of %d tokens a row", kv.max_pages, 1 << kv.shift);
    *any = true;
    return HX_OK;
}

HxAttend hx_attend_view(hx_ctx *ctx, const hx_kv_pool *pool, int layer, const KvView &kv, const hx_attend_args &g)
{
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
    a.k_exp = pool->k_exp; a.v_exp = pool->v_exp;
    a.q_wide = ((uintptr_t)g.q & 15) == 0 && g.q_token % 8 == 0 && g.q_head % 8 == 0;
    a.out_wide = ((uintptr_t)g.out & 7) == 0 && g.out_token % 4 == 0 && g.out_head % 4 == 0;
    return a;
}

int hx_attend_run(hx_ctx *ctx, int pool_dtype, int q_dtype, HxAttend &a, int max_len, hipStream_t stream)
{
    const bool bf16 = q_dtype == HX_BF16;
    if (pool_dtype == HX_E4M3) return bf16 ? hx_attend_bf16_e4m3(ctx, a, max_len, stream) : hx_attend_f16_e4m3(ctx, a, max_len, stream);
    if (pool_dtype == HX_E2M1) return bf16 ? hx_attend_bf16_e2m1(ctx, a, max_len, stream) : hx_attend_f16_e2m1(ctx, a, max_len, stream);
    return bf16 ? hx_attend_bf16(ctx, a, max_len, stream) : hx_attend_f16(ctx, a, max_len, stream);
}

extern "C" int hx_attend(hx_ctx *ctx, const hx_kv_pool *pool, int32_t layer, const hx_kv_seqs *seqs,
                         const hx_attend_args *args, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    KvView kv;
    bool any;
    if (int rc = hx_kv_view(ctx, pool, seqs, &kv)) return rc;
    if (int rc = hx_attend_check(ctx, pool, layer, kv, args, true, &any)) return rc;
    if (!any) return HX_OK;
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    HxAttend a = hx_attend_view(ctx, pool, layer, kv, *args);
    return hx_attend_run(ctx, pool->dtype, args->dtype, a, args->max_len, (hipStream_t)stream_);
}
