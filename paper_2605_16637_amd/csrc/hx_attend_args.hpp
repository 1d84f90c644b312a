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
    const void *zeros;           // 16 bytes of them, aligned
    bool q_wide, out_wide;       // q can be read 16 bytes at a time, out written 8
    int row_tiles, splits;       // parts of a row tile's keys, at most
    int chunk;                   // tiles of keys of a part
    int *done;                   // [pair][row tile] parts that are written; 0 between launches
    float *part;                 // [workgroup][rows][dim], when splits > 1
    float2 *part_ml;             // [workgroup][rows] maximum (of s log2 e) and sum
};

// hx_attend_*.hip: queries' type, and a cache of 8 bits where the name says so.
int hx_attend_bf16(hx_ctx *ctx, HxAttend &a, int max_len, hipStream_t stream);
int hx_attend_f16(hx_ctx *ctx, HxAttend &a, int max_len, hipStream_t stream);
int hx_attend_bf16_e4m3(hx_ctx *ctx, HxAttend &a, int max_len, hipStream_t stream);
int hx_attend_f16_e4m3(hx_ctx *ctx, HxAttend &a, int max_len, hipStream_t stream);
