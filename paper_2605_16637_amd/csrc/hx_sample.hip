// One token a row from its logits: temperature, top-k, top-p, min-p, and a given uniform number.
//
// Nothing is sorted.  What stays of a row is always a prefix of its order (logit falling, number rising), so a limit is one element, the
// last that stays: it is found by adding up the row's elements in bins of the logit -- counts for top-k, weights for top-p --, then the
// elements of the bin where the limit falls, in finer bins where they are many.  The token is found the same way in the
// order of the numbers.  Weights are whole numbers of 2^-q of the largest (q from 42 to 61 with the row's length, so that a row's sum
// stays below 2^62): sums do not depend on the order they are added in, and no limit on how rounding went.
#include "hx_serve.hpp"

namespace {

constexpr int SA_THREADS = 1024;
constexpr int SA_WAVES = SA_THREADS / HX_WAVE;
constexpr int SA_BINS = 128, SA_COLS = 32;        // a bin's sum lies in 32 places, a lane's by its number: lanes of a wavefront seldom meet
constexpr int SA_LIST = 256;                      // elements of the limit's bin that are compared with each other

struct SampleArgs {
    int n_rows, n_vocab, qbits;
    const void *logits;
    int64_t row_stride;
    const float *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p, *u;
    int32_t *token;
    float *logprob;
    int32_t *n_kept;
    int32_t *status;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__bf16 x) { return (float)x; }
__device__ __forceinline__ float to_float(_Float16 x) { return (float)x; }

__device__ __forceinline__ bool is_nan(float x) { return (__float_as_uint(x) & 0x7fffffffu) > 0x7f800000u; }

// unsigned keys in the order of the numbers; the two zeros are one
__device__ __forceinline__ uint32_t key_of(float x)
{
    uint32_t b = __float_as_uint(x);
    b = b == 0x80000000u ? 0u : b;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
constexpr uint32_t KEY_BARRED = 0x007fffffu;       // of -infinity; a NaN's is made the same

// 2^z for z <= 0, to 2^-50 of it: the whole part by the exponent, the rest, |f| <= 1/2, by the series of exp(f ln 2) to f^12
__device__ __forceinline__ double exp2_neg(double z)
{
    const double n = __builtin_rint(z), f = z - n;
    double p = 2.5678435993488205e-11;                        // ln2^12 / 12!
    p = __builtin_fma(p, f, 4.4455382718708116e-10);
    p = __builtin_fma(p, f, 7.0549116208011233e-09);
    p = __builtin_fma(p, f, 1.0178086009239699e-07);
    p = __builtin_fma(p, f, 1.3215486790144307e-06);
    p = __builtin_fma(p, f, 1.5252733804059841e-05);
    p = __builtin_fma(p, f, 1.5403530393381609e-04);
    p = __builtin_fma(p, f, 1.3333558146428443e-03);
    p = __builtin_fma(p, f, 9.6181291076284772e-03);
    p = __builtin_fma(p, f, 5.5504108664821580e-02);
    p = __builtin_fma(p, f, 2.4022650695910072e-01);
    p = __builtin_fma(p, f, 6.9314718055994531e-01);
    p = __builtin_fma(p, f, 1.0);
    return n < -1000.0 ? 0.0 : __builtin_ldexp(p, (int)n);
}

// floor(f * w) for 0 <= f < 1; *rest: whether something was cut off
__device__ __forceinline__ uint64_t scaled(float f, uint64_t w, bool *rest)
{
    const uint32_t b = __float_as_uint(f), e = b >> 23;
    const uint64_t m = (b & 0x7fffffu) | (e ? 0x800000u : 0u);
    const int shift = 150 - (int)(e ? e : 1);               // f = m 2^-shift, shift >= 24
    const uint64_t lo = m * w, hi = __umul64hi(m, w);
    if (shift >= 128) { *rest = (lo | hi) != 0; return 0; }
    if (shift >= 64) {
        const int s = shift - 64;
        *rest = lo != 0 || (s && (hi & ((1ull << s) - 1)) != 0);
        return hi >> s;
    }
    *rest = (lo & ((1ull << shift) - 1)) != 0;
    return hi << (64 - shift) | lo >> shift;
}

struct Shared {
    uint64_t hist[SA_BINS * SA_COLS];          // and the sums of locate()
    uint64_t wave[SA_WAVES];
    uint32_t wmin[SA_WAVES], wmax[SA_WAVES];
    uint32_t key[SA_LIST];
    int idx[SA_LIST];
    uint64_t mass[SA_LIST];
    uint64_t r64[2];
    int r32[4];
};

template <typename E>
struct Row {
    const E *p;
    int n, skip;              // elements; those of the first 16 bytes that lie before the row
    int per;                  // pieces of a wavefront, a multiple of 64
    int pieces;
    static constexpr int EACH = 16 / sizeof(E);      // elements of a piece

    __device__ void set(const E *at, int count)
    {
        p = at;
        n = count;
        skip = (int)(((uintptr_t)at & 15) / sizeof(E));
        pieces = (int)(((int64_t)n + skip + EACH - 1) / EACH);
        const int64_t w = ((int64_t)pieces + SA_WAVES - 1) / SA_WAVES;
        per = (int)((w + HX_WAVE - 1) / HX_WAVE * HX_WAVE);
    }
    // The elements of piece c: their keys, KEY_BARRED for what is not of the row.
    __device__ __forceinline__ void keys(int c, uint32_t *k) const
    {
        const int64_t first = (int64_t)c * EACH - skip;
        if (first >= 0 && first + EACH <= n) {
            struct alignas(16) Piece { E x[EACH]; };
            const Piece v = *(const Piece *)(p + first);
#pragma unroll
            for (int j = 0; j < EACH; ++j) k[j] = key(to_float(v.x[j]));
        } else {
#pragma unroll
            for (int j = 0; j < EACH; ++j) k[j] = first + j >= 0 && first + j < n ? key(to_float(p[first + j])) : KEY_BARRED;
        }
    }
    static __device__ __forceinline__ uint32_t key(float x) { return is_nan(x) ? KEY_BARRED : key_of(x); }
    __device__ __forceinline__ int index(int c, int j) const { return c * EACH - skip + j; }
    // f(piece, its keys) for all of this wavefront's, all lanes together
    template <typename F>
    __device__ __forceinline__ void each(F f) const
    {
        const int lane = threadIdx.x & 63, c0 = (threadIdx.x >> 6) * per;
        for (int it = 0; it < per; it += HX_WAVE) {
            const int c = c0 + it + lane;
            uint32_t k[EACH];
            if (c < pieces) keys(c, k);
            else
#pragma unroll
                for (int j = 0; j < EACH; ++j) k[j] = KEY_BARRED;
            f(c, k, it / HX_WAVE);
        }
    }
};

__device__ __forceinline__ uint64_t wave_sum(uint64_t x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

// What stays: elements before the last one, and that one.
struct Limit {
    uint32_t key;             // of the last that stays
    int idx;                  // its number: of equal keys those up to it stay
    __device__ __forceinline__ bool holds(uint32_t k, int i) const { return k > key || (k == key && i <= idx); }
};

// The lowest element at which the sum of `mass` in the order of the numbers exceeds target(total); -1: nowhere.
template <typename E, typename M, typename W>
__device__ int locate(const Row<E> &row, Shared &s, M mass, W target, uint64_t *total)
{
    constexpr int EACH = Row<E>::EACH;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, iters = row.per / HX_WAVE;
    __syncthreads();
    row.each([&](int c, const uint32_t *k, int it) {
        uint64_t x = 0;
#pragma unroll
        for (int j = 0; j < EACH; ++j) x += k[j] > KEY_BARRED ? mass(k[j], row.index(c, j)) : 0;
        x = wave_sum(x);
        if (lane == 0) s.hist[w * iters + it] = x;
    });
    if (tid == 0) s.r32[0] = -1;
    __syncthreads();
    // the step of 64 pieces at which it is exceeded: by the first wavefront
    if (w == 0) {
        uint64_t all = 0;
        for (int i = lane; i < SA_WAVES * iters; i += HX_WAVE) all += s.hist[i];
        all = wave_sum(all);
        const uint64_t want = target(all);
        uint64_t before = 0;
        int at = -1;
        for (int i0 = 0; i0 < SA_WAVES * iters && at < 0; i0 += HX_WAVE) {
            uint64_t x = i0 + lane < SA_WAVES * iters ? s.hist[i0 + lane] : 0, sum = x;
#pragma unroll
            for (int d = 1; d < HX_WAVE; d <<= 1) {
                const uint64_t y = __shfl_up(sum, d);
                if (lane >= d) sum += y;
            }
            const unsigned long long m = __builtin_amdgcn_ballot_w64(before + sum > want);
            if (m) {
                const int l = __builtin_ctzll(m);
                at = i0 + l;
                before += __shfl(sum - x, l);
            } else before += __shfl(sum, 63);
        }
        if (at >= 0) {
            const int c = (at / iters) * row.per + (at % iters) * HX_WAVE + lane;
            uint32_t k[EACH];
            uint64_t q[EACH], x = 0;
            if (c < row.pieces) row.keys(c, k);
            else
#pragma unroll
                for (int j = 0; j < EACH; ++j) k[j] = KEY_BARRED;
#pragma unroll
            for (int j = 0; j < EACH; ++j) { q[j] = k[j] > KEY_BARRED ? mass(k[j], row.index(c, j)) : 0; x += q[j]; }
            uint64_t sum = x;
#pragma unroll
            for (int d = 1; d < HX_WAVE; d <<= 1) {
                const uint64_t y = __shfl_up(sum, d);
                if (lane >= d) sum += y;
            }
            uint64_t run = before + sum - x;
            int found = -1;
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                run += q[j];
                if (found < 0 && run > want) found = row.index(c, j);
            }
            const unsigned long long m = __builtin_amdgcn_ballot_w64(found >= 0);
            if (m && lane == __builtin_ctzll(m)) s.r32[0] = found;
        }
        if (lane == 0) s.r64[0] = all;
    }
    __syncthreads();
    const int got = s.r32[0];
    *total = s.r64[0];
    __syncthreads();
    return got;
}

// The last element that stays of those for which `in` holds, in the order (logit falling, number rising): the one at which the sum of
// `mass` reaches want(total).  false: all stay, or none is there.
template <typename E, typename I, typename M, typename W>
__device__ bool find_limit(const Row<E> &row, Shared &s, float top, float reach, I in, M mass, W want, Limit *out)
{
    constexpr int EACH = Row<E>::EACH;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    // first bins: by how far a logit lies below the largest, the last for all that lie beyond `reach`
    const float unit = reach > 0.0f ? (SA_BINS - 1) / reach : 0.0f;
    uint32_t k_low = KEY_BARRED + 1, k_high = 0xffffffffu;       // keys still in question
    int shift = -1;                                              // -1: first bins; else bins of (k_high - key) >> shift
    uint64_t before = 0, limit = 0;
    auto bin_of = [&](uint32_t k) {
        if (shift >= 0) return (int)((k_high - k) >> shift);
        const float d = fminf((top - of_key(k)) * unit, (float)(SA_BINS - 1));
        return of_key(k) == top ? 0 : (int)d;
    };
    for (bool first = true;; first = false) {
        __syncthreads();
        for (int i = tid; i < SA_BINS * SA_COLS; i += SA_THREADS) s.hist[i] = 0;
        __syncthreads();
        row.each([&](int c, const uint32_t *k, int) {
#pragma unroll
            for (int j = 0; j < EACH; ++j)
                if (k[j] >= k_low && k[j] <= k_high && in(k[j], row.index(c, j)))
                    if (const uint64_t x = mass(k[j])) atomicAdd((unsigned long long *)&s.hist[bin_of(k[j]) * SA_COLS + (lane & (SA_COLS - 1))], (unsigned long long)x);
        });
        __syncthreads();
        // a thread a bin adds its places up, the first wavefront then the bins
        if (tid < SA_BINS) {
            uint64_t x = 0;
            for (int i = 0; i < SA_COLS; ++i) x += s.hist[tid * SA_COLS + ((i + tid) & (SA_COLS - 1))];
            s.mass[tid] = x;
        }
        __syncthreads();
        if (w == 0) {
            const uint64_t x0 = s.mass[2 * lane], x1 = s.mass[2 * lane + 1];
            uint64_t sum = x0 + x1;
#pragma unroll
            for (int d = 1; d < HX_WAVE; d <<= 1) {
                const uint64_t y = __shfl_up(sum, d);
                if (lane >= d) sum += y;
            }
            const uint64_t all = __shfl(sum, 63);
            uint64_t lim = limit;
            if (first) lim = want(all);
            const uint64_t b0 = before + sum - x0 - x1, b1 = b0 + x0;
            if (lane == 0) { s.r32[1] = -1; s.r64[1] = lim; }
            if (b0 < lim && lim <= b0 + x0) { s.r32[1] = 2 * lane; s.r64[0] = b0; }
            if (b1 < lim && lim <= b1 + x1) { s.r32[1] = 2 * lane + 1; s.r64[0] = b1; }
        }
        if (tid == 0) s.r32[2] = 0;
        __syncthreads();
        const int bin = s.r32[1];
        limit = s.r64[1];
        if (bin < 0) return false;
        before = s.r64[0];
        // the elements of that bin
        uint32_t lo = 0xffffffffu, hi = 0;
        row.each([&](int c, const uint32_t *k, int) {
#pragma unroll
            for (int j = 0; j < EACH; ++j)
                if (k[j] >= k_low && k[j] <= k_high && in(k[j], row.index(c, j)) && bin_of(k[j]) == bin)
                    if (const uint64_t x = mass(k[j])) {
                        lo = k[j] < lo ? k[j] : lo;
                        hi = k[j] > hi ? k[j] : hi;
                        const int at = atomicAdd(&s.r32[2], 1);
                        if (at < SA_LIST) { s.key[at] = k[j]; s.idx[at] = row.index(c, j); s.mass[at] = x; }
                    }
        });
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const uint32_t a = __shfl_xor(lo, d), b = __shfl_xor(hi, d);
            lo = a < lo ? a : lo;
            hi = b > hi ? b : hi;
        }
        if (lane == 0) { s.wmin[w] = lo; s.wmax[w] = hi; }
        __syncthreads();
        const int count = s.r32[2];
        for (int i = 0; i < SA_WAVES; ++i) {
            lo = s.wmin[i] < lo ? s.wmin[i] : lo;
            hi = s.wmax[i] > hi ? s.wmax[i] : hi;
        }
        if (count <= SA_LIST) {
            if (tid < count) {
                const uint32_t k = s.key[tid];
                const int i = s.idx[tid];
                uint64_t b = before;
                for (int j = 0; j < count; ++j) {
                    const uint32_t kj = s.key[j];
                    b += kj > k || (kj == k && s.idx[j] < i) ? s.mass[j] : 0;
                }
                if (b < limit && limit <= b + s.mass[tid]) { s.r32[3] = i; s.r64[0] = k; }
            }
            __syncthreads();
            out->key = (uint32_t)s.r64[0];
            out->idx = s.r32[3];
            __syncthreads();
            return true;
        }
        if (lo == hi) {
            // all equal: the first so many by their numbers
            const uint64_t x = mass(lo), stay = (limit - before + x - 1) / x;
            uint64_t all;
            out->key = lo;
            out->idx = locate(row, s, [&](uint32_t k, int i) -> uint64_t { return k == lo && in(k, i); },
                              [&](uint64_t) -> uint64_t { return stay - 1; }, &all);
            return true;
        }
        k_low = lo;
        k_high = hi;
        shift = 0;
        while (((hi - lo) >> shift) >= SA_BINS) ++shift;
    }
}

template <typename E>
__global__ __launch_bounds__(SA_THREADS) void hx_sample_kernel(SampleArgs a)
{
    constexpr int EACH = Row<E>::EACH;
    __shared__ Shared s;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    Row<E> row;
    row.set((const E *)a.logits + (int64_t)r * a.row_stride, a.n_vocab);

    const float T = a.temperature ? a.temperature[r] : 1.0f, p = a.top_p ? a.top_p[r] : 1.0f, mp = a.min_p ? a.min_p[r] : 0.0f, u = a.u[r];
    const int k = a.top_k ? a.top_k[r] : 0;
    const bool fine = !is_nan(T) && !is_nan(p) && !is_nan(mp) && !is_nan(u) && T >= 0.0f && __float_as_uint(T) != 0x7f800000u && mp >= 0.0f && mp <= 1.0f &&
                      u >= 0.0f && u < 1.0f;

    // the largest and the least logit that are not barred
    uint32_t hi = 0, lo = 0xffffffffu;
    bool nan = false;
    row.each([&](int c, const uint32_t *kk, int) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            hi = kk[j] > hi ? kk[j] : hi;
            lo = kk[j] > KEY_BARRED && kk[j] < lo ? kk[j] : lo;
        }
    });
    // a NaN is told by its bits
    {
        const int lane_c0 = w * row.per + lane;
        for (int it = 0; it < row.per; it += HX_WAVE) {
            const int c = lane_c0 + it;
            for (int j = 0; j < EACH; ++j) {
                const int i = row.index(c, j);
                if (c < row.pieces && i >= 0 && i < row.n) nan |= is_nan(to_float(row.p[i]));
            }
        }
    }
    if (nan || (!fine && tid == 0)) hx_raise(a.status, HX_ERR_INVALID_ARG);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const uint32_t x = __shfl_xor(hi, d), y = __shfl_xor(lo, d);
        hi = x > hi ? x : hi;
        lo = y < lo ? y : lo;
    }
    if (lane == 0) { s.wmax[w] = hi; s.wmin[w] = lo; }
    __syncthreads();
    for (int i = 0; i < SA_WAVES; ++i) {
        hi = s.wmax[i] > hi ? s.wmax[i] : hi;
        lo = s.wmin[i] < lo ? s.wmin[i] : lo;
    }
    __syncthreads();
    if (!fine || hi <= KEY_BARRED) {
        if (tid == 0) {
            a.token[r] = -1;
            if (a.logprob) a.logprob[r] = -__builtin_inff();
            if (a.n_kept) a.n_kept[r] = 0;
        }
        return;
    }
    const float top = of_key(hi);
    uint64_t all;
    if (T == 0.0f) {
        const int t = locate(row, s, [&](uint32_t kk, int) -> uint64_t { return kk == hi; }, [](uint64_t) -> uint64_t { return 0; }, &all);
        if (tid == 0) {
            a.token[r] = t;
            if (a.logprob) a.logprob[r] = 0.0f;
            if (a.n_kept) a.n_kept[r] = 1;
        }
        return;
    }
    const bool boundless = hi == 0xff800000u;              // +infinity takes all the weight
    const double inv = 1.4426950408889634 / (double)T, one = __builtin_ldexp(1.0, a.qbits);
    auto weight = [&](uint32_t kk) -> double {
        if (boundless) return kk == hi ? 1.0 : 0.0;
        return exp2_neg(((double)of_key(kk) - (double)top) * inv);
    };
    auto whole = [&](double x) -> uint64_t { return (uint64_t)(x * one + 0.5); };

    Limit lim{KEY_BARRED + 1, 0x7fffffff};                 // all that are not barred
    const float span = top - of_key(lo);
    if (k > 0)
        find_limit(row, s, top, fminf(span, 32.0f), [](uint32_t, int) { return true; }, [](uint32_t) -> uint64_t { return 1; },
                   [&](uint64_t n) -> uint64_t { return (uint64_t)k < n ? (uint64_t)k : ~0ull; }, &lim);
    if (p < 1.0f) {
        const Limit of = lim;
        find_limit(row, s, top, fminf(span, 40.0f * T), [&](uint32_t kk, int i) { return of.holds(kk, i); }, [&](uint32_t kk) { return whole(weight(kk)); },
                   [&](uint64_t n) -> uint64_t {
                       if (p <= 0.0f) return 1;
                       bool rest;
                       const uint64_t x = scaled(p, n, &rest) + 1;       // one more than the floor ..
                       const uint64_t up = rest ? x : x - 1;             // .. unless nothing was cut off
                       return up ? up : 1;
                   }, &lim);
    }
    const double min_w = mp;
    const int t = locate(row, s, [&](uint32_t kk, int i) -> uint64_t {
        if (!lim.holds(kk, i)) return 0;
        const double x = weight(kk);
        return x >= min_w ? whole(x) : 0;
    }, [&](uint64_t n) -> uint64_t { bool rest; return scaled(u, n, &rest); }, &all);
    if (tid == 0) a.token[r] = t;
    if (a.n_kept || a.logprob) {
        int mine = 0;
        if (a.n_kept)
            row.each([&](int c, const uint32_t *kk, int) {
#pragma unroll
                for (int j = 0; j < EACH; ++j) mine += kk[j] > KEY_BARRED && lim.holds(kk[j], row.index(c, j)) && (min_w <= 0.0 || weight(kk[j]) >= min_w);
            });
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) mine += __shfl_xor(mine, d);
        __syncthreads();
        if (lane == 0) s.wmin[w] = (uint32_t)mine;
        __syncthreads();
        if (tid == 0) {
            int n = 0;
            for (int i = 0; i < SA_WAVES; ++i) n += (int)s.wmin[i];
            if (a.n_kept) a.n_kept[r] = n;
            if (a.logprob) {
                const float x = to_float(row.p[t]);
                const double d = boundless ? 0.0 : ((double)x - (double)top) / (double)T;
                a.logprob[r] = (float)(d - (log((double)all) - a.qbits * 0.6931471805599453));
            }
        }
    }
}

}  // namespace

extern "C" int hx_sample(hx_ctx *ctx, int32_t n_rows, int32_t n_vocab, int32_t dtype, const void *logits, int64_t row_stride,
                         const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p, const float *u,
                         int32_t *token, float *logprob, int32_t *n_kept, void *stream_)
{
    if (!ctx) return HX_ERR_INVALID_ARG;
    HX_REQUIRE(ctx, n_rows >= 0 && n_vocab >= 0, HX_ERR_INVALID_ARG, "negative size");
    HX_REQUIRE(ctx, n_vocab <= HX_MAX_VOCAB, HX_ERR_SHAPE, "%d logits a row, beyond %d", n_vocab, HX_MAX_VOCAB);
    HX_REQUIRE(ctx, dtype == HX_F32 || dtype == HX_BF16 || dtype == HX_F16, HX_ERR_INVALID_ARG, "logits of type %d", dtype);
    if (n_rows == 0) return HX_OK;
    HX_REQUIRE(ctx, n_vocab > 0, HX_ERR_INVALID_ARG, "rows without a logit");
    HX_REQUIRE(ctx, logits && u && token, HX_ERR_INVALID_ARG, "NULL array");
    HX_REQUIRE(ctx, ((uintptr_t)logits & (hx_type_size(dtype) - 1)) == 0, HX_ERR_INVALID_ARG, "logits are not aligned to their type");
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    hipStream_t stream = (hipStream_t)stream_;
    int bits = 0;
    while (((int64_t)1 << bits) < n_vocab) ++bits;
    SampleArgs a{n_rows, n_vocab, 62 - bits - 1, logits, row_stride, temperature, top_k, top_p, min_p, u, token, logprob, n_kept, ctx->d_status};
    if (dtype == HX_F32) hx_sample_kernel<float><<<n_rows, SA_THREADS, 0, stream>>>(a);
    else if (dtype == HX_BF16) hx_sample_kernel<__bf16><<<n_rows, SA_THREADS, 0, stream>>>(a);
    else hx_sample_kernel<_Float16><<<n_rows, SA_THREADS, 0, stream>>>(a);
    return hx_check_launch(ctx, "hx_sample_kernel");
}
