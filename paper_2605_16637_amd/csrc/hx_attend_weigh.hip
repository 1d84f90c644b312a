// The weights that attention has given each cached token, summed over queries and heads.
#include "hx_attend_common.hpp"

namespace {

constexpr int WG_THREADS = 256, WG_WAVES = WG_THREADS / 64;

struct WeighArgs {
    AttendArgs a;
    float *weight;
    int64_t pitch;               // of a row's weights
    int each;                    // workgroups of a sequence
};

// Whether the row of entry i is listed before it too; all threads take part.
__device__ __forceinline__ bool row_before(const AttendArgs &a, int i)
{
    if (!a.row) return false;
    const int mine = a.row[i];
    bool hit = false;
    for (int k = threadIdx.x; k < i; k += WG_THREADS) hit |= a.row[k] == mine;
    return __syncthreads_or(hit);
}

// A wavefront takes 16 BLOCKS keys of a sequence and all heads: its weights are its own, and their sums need no other's.  The keys of a head go from memory
// into the registers of the product with 16 rows (queries x query heads of the KV head) at a time; the next head's are under way while
// weights are worked out.
template <typename E, int BITS, int D, int BLOCKS>
__global__ __launch_bounds__(WG_THREADS) void hx_weigh_kernel(WeighArgs w)
{
    using X8 = typename Types<E>::x8;
    using Keys = KeyPieces<BITS, D>;
    using KPiece = typename Keys::Piece;
    constexpr int ROW_BYTES = ROW<BITS, D>, KEYS = 16 * BLOCKS, TILE = KEYS * WG_WAVES;
    extern __shared__ __align__(16) char smem[];
    int *s_depth = (int *)smem + HX_MAX_DRAFTS;
    uint32_t *s_anc = (uint32_t *)(s_depth + HX_MAX_DRAFTS);
    const AttendArgs &a = w.a;
    const KvView &kv = a.kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), quad = lane >> 4, col = lane & 15;
    const int i = blockIdx.x % a.n, part = blockIdx.x / a.n;
    const Seq sq = sequence(a, i * kv.n_heads);
    const Extent ex = extent<TILE>(a, sq, 0, sq.nq - 1);
    if (!sq.ok) { if (tid == 0 && part == 0 && (!sq.there || sq.nq > 0)) hx_raise(kv.status, HX_ERR_INDEX); return; }
    if (sq.nq == 0 || part >= ex.n) return;
    if (row_before(a, i)) { if (tid == 0 && part == 0) hx_raise(kv.status, HX_ERR_INDEX); return; }
    const bool tree = a.parent != nullptr;
    if (tree) plant(a, sq, (int *)smem, s_depth, s_anc);
    const int r = a.row ? a.row[i] : i, rows = sq.nq * a.group, row_tiles = (rows + 15) / 16;
    const int64_t page_bytes = ((int64_t)kv.n_heads << kv.shift) * ROW_BYTES, head_bytes = (int64_t)ROW_BYTES << kv.shift;
    const int64_t here = (int64_t)a.layer * kv.n_pages * page_bytes;
    const char *k_at = (const char *)kv.k + here;
    const uint8_t *ke_at = BITS == 4 ? a.k_exp + here / 16 : nullptr;
    for (int tile = part; tile < ex.n; tile += w.each) {
        const int y0 = (tile < ex.sink_tiles ? tile : tile - ex.sink_tiles + ex.lo_tile) * TILE + wave * KEYS;
        // lane x looks up key x; what is not there reads the pool's first page, and counts for nothing
        int page = -1;
        {
            const int y = y0 + (lane & (KEYS - 1));
            if (y < ex.hi && (y >= ex.lo || y < a.n_sink)) page = sq.table[y >> kv.shift];
            page = in_pool(kv, page);
        }
        const uint64_t there = __builtin_amdgcn_ballot_w64(page >= 0) & (KEYS == 64 ? ~0ull : (1ull << (KEYS & 63)) - 1);
        if (there == 0) continue;
        int64_t at[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const int p = __shfl(page, b * 16 + col), y = y0 + b * 16 + col;
            at[b] = (p < 0 ? 0 : p * page_bytes + (y & ((1 << kv.shift) - 1)) * ROW_BYTES) + quad * Keys::BYTES;
        }
        KPiece rk[BLOCKS][Keys::LOADS];
        uint8_t ek[BLOCKS][Keys::LOADS];
        auto fetch_k = [&](int head) {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int l = 0; l < Keys::LOADS; ++l) {
                    rk[b][l] = *(const KPiece *)(k_at + at[b] + head * head_bytes + l * 64);
                    if constexpr (BITS == 4) ek[b][l] = ke_at[(at[b] + head * head_bytes + l * 64) / 16];
                }
        };
        X8 qf[D / 32];
        float lse;
        auto fetch_q = [&](int head, int rt) {
            const int row = rt * 16 + col;
            const bool in = row < rows;
            const int t = in ? row / a.group : 0, qhead = head * a.group + (in ? row % a.group : 0);
            const E *q = (const E *)a.q + (int64_t)(sq.q0 + t) * a.q_token + (int64_t)qhead * a.q_head;
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                const int d = Keys::place(s, quad);
                X8 x = {};
                if (in) {
                    if (a.q_wide) x = *(const X8 *)(q + d);
                    else
#pragma unroll
                        for (int j = 0; j < 8; ++j) x[j] = q[d + j];
                }
                qf[s] = x;
            }
            lse = in ? a.lse[(int64_t)(sq.q0 + t) * a.n_heads + qhead] : __builtin_inff();
        };
        float sum[BLOCKS][4] = {};
        fetch_k(0);
        fetch_q(0, 0);
        for (int head = 0; head < kv.n_heads; ++head) {
            const float k_unit = a.k_scale ? a.k_scale[a.layer * kv.n_heads + head] : 1.0f, sc = a.scale * k_unit;
            // as in attention the factor is no 0, and its sign the query's: a score of -infinity stays one
            const float c = copysignf(fmaxf(fabsf(sc), 1e-37f), sc);
            for (int rt = 0; rt < row_tiles; ++rt) {
                f32x4 s[BLOCKS] = {};
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int l = 0; l < Keys::LOADS; ++l)
#pragma unroll
                        for (int j = 0; j < Keys::EACH; ++j) s[b] = mfma16(Keys::template operand<E>(rk[b][l], ek[b][l], j), qf[Keys::EACH * l + j], s[b]);
                const float mine = lse;
                if (rt + 1 < row_tiles) fetch_q(head, rt + 1);
                else if (head + 1 < kv.n_heads) {
                    fetch_k(head + 1);
                    fetch_q(head + 1, 0);
                }
                const int t = (rt * 16 + col) / a.group, t_last = (rt * 16 + 15) / a.group, last = sq.base + (t_last < sq.nq ? t_last : sq.nq - 1);
                const int first = tree ? sq.base - 1 : sq.base + rt * 16 / a.group, end = y0 + KEYS - 1;
                const bool counts = rt * 16 + col < rows && __builtin_fabsf(mine) < __builtin_inff();
                const bool whole = there == (KEYS == 64 ? ~0ull : (1ull << (KEYS & 63)) - 1) && end <= first &&
                                   (a.window <= 0 || end < a.n_sink || (tree ? sq.len : last) - y0 < a.window);
                if (whole) {
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const float p = __builtin_amdgcn_exp2f(fmaf(s[b][x], c, -mine) * LOG2E);
                            sum[b][x] += counts ? p : 0.0f;
                        }
                } else {
                    const Sight view = sight(a, sq, t, s_depth, s_anc);
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int k = b * 16 + quad * 4 + x;
                            const float p = __builtin_amdgcn_exp2f(fmaf(s[b][x], c, -mine) * LOG2E);
                            sum[b][x] += counts && ((there >> k) & 1) && view.sees(y0 + k) ? p : 0.0f;
                        }
                }
            }
        }
        // a key's sums lie over 16 lanes
        float *to = w.weight + r * w.pitch;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int d = 8; d > 0; d >>= 1) sum[b][x] += __shfl_xor(sum[b][x], d);
            const int k = b * 16 + quad * 4 + col;
            if (col < 4 && ((there >> k) & 1)) to[y0 + k] += col == 0 ? sum[b][0] : col == 1 ? sum[b][1] : col == 2 ? sum[b][2] : sum[b][3];
        }
    }
}

template <typename E, int BITS, int D>
int launch(hx_ctx *ctx, WeighArgs &w, int max_len, hipStream_t stream)
{
    constexpr int BLOCKS = 2;
    const int TILE = 16 * BLOCKS * WG_WAVES;
    int64_t reach = max_len;
    const HxAttend &a = w.a;
    if (a.window > 0 && reach > (int64_t)a.window + a.n_sink + a.max_q) reach = (int64_t)a.window + a.n_sink + a.max_q;
    const int64_t tiles = (reach + TILE - 1) / TILE + 2, most = hx_most_groups(WG_THREADS) / a.n;
    w.each = (int)(tiles < most ? tiles : most);
    const int lds = a.parent ? HX_MAX_DRAFTS * 4 + TREE_BYTES : 0;
    hx_weigh_kernel<E, BITS, D, BLOCKS><<<(int)((int64_t)w.each * a.n), WG_THREADS, lds, stream>>>(w);
    return hx_check_launch(ctx, "hx_weigh_kernel");
}

template <typename E, int BITS>
int by_dim(hx_ctx *ctx, WeighArgs &w, int max_len, hipStream_t stream)
{
    if (w.a.kv.dim == 64) return launch<E, BITS, 64>(ctx, w, max_len, stream);
    if (w.a.kv.dim == 128) return launch<E, BITS, 128>(ctx, w, max_len, stream);
    return launch<E, BITS, 256>(ctx, w, max_len, stream);
}

template <typename E>
int by_type(hx_ctx *ctx, int pool_dtype, WeighArgs &w, int max_len, hipStream_t stream)
{
    if (pool_dtype == HX_E4M3) return by_dim<E, 8>(ctx, w, max_len, stream);
    if (pool_dtype == HX_E2M1) return by_dim<E, 4>(ctx, w, max_len, stream);
    return by_dim<E, 16>(ctx, w, max_len, stream);
}

}  // namespace

extern "C" int hx_kv_weigh(hx_ctx *ctx, const hx_kv_pool *pool, int32_t layer, const hx_kv_seqs *seqs,
                           const hx_attend_args *args, float *weight, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    KvView kv;
    bool any;
    if (int rc = hx_kv_view(ctx, pool, seqs, &kv)) return rc;
    if (int rc = hx_attend_check(ctx, pool, layer, kv, args, false, &any)) return rc;
    if (!any) return HX_OK;
    HX_REQUIRE(ctx, args->lse && weight, HX_ERR_INVALID_ARG, "NULL lse or weights");
    HX_REQUIRE(ctx, (((uintptr_t)args->lse | (uintptr_t)weight) & 3) == 0, HX_ERR_INVALID_ARG, "lse or weights are not aligned to their type");
    HX_REQUIRE(ctx, args->n <= hx_most_groups(WG_THREADS), HX_ERR_SHAPE, "%d sequences in one call", args->n);
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    WeighArgs w{hx_attend_view(ctx, pool, layer, kv, *args), weight, (int64_t)kv.max_pages << kv.shift, 1};
    return args->dtype == HX_BF16 ? by_type<__bf16>(ctx, pool->dtype, w, args->max_len, (hipStream_t)stream_)
                                  : by_type<_Float16>(ctx, pool->dtype, w, args->max_len, (hipStream_t)stream_);
}
