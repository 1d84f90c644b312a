// What attention's entry point hands to its kernels.
#pragma once

#include "hx_serve.hpp"

// A call's arguments as its kernels take them.
struct HxAttend {
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
    const uint8_t *k_exp, *v_exp;
    const int32_t *picked;       // [query][KV head][picked_pages] pages chosen for each, or NULL: then n = n_q, and each is a sequence
    const int32_t *picked_len;   // [query][KV head] the place of the query's own token among the chosen pages' + 1
    int picked_pages;
    bool room_only;              // scratch is asked for, nothing launched
    const void *zeros;           // 16 bytes of them, aligned
    bool q_wide, out_wide;       // q can be read 16 bytes at a time, out written 8
    int row_tiles, splits;       // parts of a row tile's keys, at most
    int chunk;                   // tiles of keys of a part
    int *done;                   // [pair][row tile] parts that are written; 0 between launches
    float *part;                 // [workgroup][rows][dim], when splits > 1
    float2 *part_ml;             // [workgroup][rows] maximum (of s log2 e) and sum
};

// hx_attend_*.hip: queries' type, and a cache of 8 or 4 bits where the name says so.
int hx_attend_bf16(hx_ctx *ctx, HxAttend &a, int max_len, hipStream_t stream);
int hx_attend_f16(hx_ctx *ctx, HxAttend &a, int max_len, hipStream_t stream);
int hx_attend_bf16_e4m3(hx_ctx *ctx, HxAttend &a, int max_len, hipStream_t stream);
int hx_attend_f16_e4m3(hx_ctx *ctx, HxAttend &a, int max_len, hipStream_t stream);
int hx_attend_bf16_e2m1(hx_ctx *ctx, HxAttend &a, int max_len, hipStream_t stream);
int hx_attend_f16_e2m1(hx_ctx *ctx, HxAttend &a, int max_len, hipStream_t stream);
int hx_attend_run(hx_ctx *ctx, int pool_dtype, int q_dtype, HxAttend &a, int max_len, hipStream_t stream);       // whichever of these it is

// hx_attend.hip: the checks of a call's arguments (any: whether there is anything to do), and the arguments as the kernels take them.
int hx_attend_check(hx_ctx *ctx, const hx_kv_pool *pool, int layer, const KvView &kv, const hx_attend_args *args, bool with_out, bool *any);
HxAttend hx_attend_view(hx_ctx *ctx, const hx_kv_pool *pool, int layer, const KvView &kv, const hx_attend_args &args);
