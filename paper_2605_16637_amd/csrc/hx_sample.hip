// One token a row from its logits: temperature, top-k, top-p, min-p, and a given uniform number.
//
// Nothing is sorted.  What stays of a row is always a prefix of its order (logit falling, number rising), so a limit is one element, the
// last that stays: it is found by adding up the row's elements in bins of the logit -- counts for top-k, weights for top-p --, then the
// elements of the bin where the limit falls, in finer bins where they are many.  The token is found the same way in the
// order of the numbers.  Weights are whole numbers of 2^-q of the largest (q = 42 to 50 by the row's length, so that a row's sum
// stays below 2^62): sums do not depend on the order they are added in, and no limit on how rounding went.
//
// A workgroup a row; a row is read three to five times (from the caches after the first).  Bound by instructions, of which a weight takes
// 26, 14 of them in 64 bits; where top-k or min-p leave few elements, only these have weights.  256 rows of 131071 bf16 logits (67 MB; one
// reading takes 14 us at a copy's rate): greedy 45 us, temperature alone 67, top-k 50 49, top-p 0.9 163.  One row of 32000 fp32 on one CU: 16,
// 23, 25 and 53 us.
#include "hx_serve.hpp"

namespace {

constexpr int SA_THREADS = 1024;
constexpr int SA_WAVES = SA_THREADS / HX_WAVE;
constexpr int SA_UNROLL = 4;                      // pieces of 16 bytes a lane has under way, and adds up before the wavefront does
constexpr int SA_STEP = SA_UNROLL * HX_WAVE;
constexpr int SA_BINS = 1408, SA_COLS = 4;        // 32 bins to a factor of 2 in weight, 44 factors; a bin's sum lies in 4 places, a lane's by its number
constexpr int SA_LIST = 1792;                     // elements of the limit's bin that are looked at in LDS
constexpr int SA_FEW = 256;                       // of them, those that are compared with each other
constexpr int SA_SHORT = 512;                     // elements that are all that can stay: what follows looks at them alone

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

__device__ __forceinline__ bool is_nan(float x) { return x != x; }

// unsigned keys in the order of the numbers; the two zeros are one
__device__ __forceinline__ uint32_t key_of(float x)
{
    uint32_t b = __float_as_uint(x);
    b = b == 0x80000000u ? 0u : b;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
constexpr uint32_t KEY_BARRED = 0x007fffffu;       // of -infinity; a NaN's is made the same
constexpr uint32_t KEY_INF = 0xff800000u;          // of +infinity; the keys beyond are no numbers

// floor(f * w) for 0 <= f < 1; *rest: whether something was cut off
__device__ __forceinline__ uint64_t scaled(float f, uint64_t w, bool *rest)
{
    const uint32_t b = __float_as_uint(f) & 0x7fffffffu, e = b >> 23;         // (f may be -0)
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
    uint32_t lkey[SA_LIST];
    int lidx[SA_LIST];
    uint4 edge[2];                             // the row's first and last 16 bytes, without what is not of the row
    double tab[32];                            // 2^(j / 32)
    uint64_t wave[SA_WAVES];
    int wmin[SA_WAVES], wmax[SA_WAVES];
    uint64_t r64[2];
    int r32[4];
};

template <typename E> struct Raw;
template <> struct Raw<float> {
    static constexpr int EACH = 4;
    static constexpr uint32_t BARRED = 0xff800000u;
    static constexpr int INF = 0x7f800000;
    // signed whole numbers in the order of the stored ones
    static __device__ __forceinline__ void extremes(const uint32_t *w, int &hi, int &lo)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = (int)w[i], s = x ^ ((x >> 31) & 0x7fffffff);
            hi = s > hi ? s : hi;
            lo = s < lo ? s : lo;
        }
    }
    static __device__ __forceinline__ float of_order(int s) { return __uint_as_float((uint32_t)(s ^ ((s >> 31) & 0x7fffffff))); }
    static __device__ __forceinline__ float get(const uint32_t *w, int j) { return __uint_as_float(w[j]); }
};
typedef short i16x2 __attribute__((ext_vector_type(2)));
template <typename E> struct Raw16 {
    static constexpr int EACH = 8;
    static __device__ __forceinline__ void extremes(const uint32_t *w, int &hi, int &lo)
    {
        i16x2 h = __builtin_bit_cast(i16x2, hi), l = __builtin_bit_cast(i16x2, lo);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const i16x2 x = __builtin_bit_cast(i16x2, w[i]), s = x ^ ((x >> 15) & (short)0x7fff);
            h = __builtin_elementwise_max(h, s);
            l = __builtin_elementwise_min(l, s);
        }
        hi = __builtin_bit_cast(int, h);
        lo = __builtin_bit_cast(int, l);
    }
};
template <> struct Raw<__bf16> : Raw16<__bf16> {
    static constexpr uint32_t BARRED = 0xff80ff80u;
    static constexpr int INF = 0x7f80;
    static __device__ __forceinline__ float of_order(int s) { return __uint_as_float((uint32_t)(s ^ ((s >> 31) & 0x7fff)) << 16); }
    static __device__ __forceinline__ float get(const uint32_t *w, int j) { return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16); }
};
template <> struct Raw<_Float16> : Raw16<_Float16> {
    static constexpr uint32_t BARRED = 0xfc00fc00u;
    static constexpr int INF = 0x7c00;
    static __device__ __forceinline__ float of_order(int s) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(s ^ ((s >> 31) & 0x7fff))); }
    static __device__ __forceinline__ float get(const uint32_t *w, int j) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[j / 2] >> (16 * (j & 1)))); }
};

// A row in pieces of 16 aligned bytes; wavefront w has the pieces w per .. (w + 1) per - 1.
template <typename E>
struct Row {
    using R = Raw<E>;
    static constexpr int EACH = R::EACH;
    const E *p;
    const uint4 *base, *edge;
    int n, skip;              // elements; those of the first piece that lie before the row
    int per, pieces;
    bool nans;                // some element is no number

    __device__ void set(const E *at, int count, uint4 *s_edge)
    {
        p = at;
        n = count;
        nans = false;
        skip = (int)(((uintptr_t)at & 15) / sizeof(E));
        base = (const uint4 *)(p - skip);
        edge = s_edge;
        pieces = (int)(((int64_t)n + skip + EACH - 1) / EACH);
        const int64_t w = ((int64_t)pieces + SA_WAVES - 1) / SA_WAVES;
        per = (int)((w + SA_STEP - 1) / SA_STEP * SA_STEP);
        if (threadIdx.x % HX_WAVE == 0 && threadIdx.x < 2 * HX_WAVE) s_edge[threadIdx.x / HX_WAVE] = by_element(threadIdx.x ? pieces - 1 : 0);
        __syncthreads();
    }
    // piece c, -infinity for what is not of the row
    __device__ __forceinline__ uint4 by_element(int c) const
    {
        const int64_t first = (int64_t)c * EACH - skip;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = R::BARRED;
#pragma unroll
        for (int j = 0; j < EACH; ++j)
            if (first + j >= 0 && first + j < n) {
                const E x = p[first + j];
                if constexpr (sizeof(E) == 4) w[j] = __float_as_uint(x);
                else {
                    const uint32_t y = __builtin_bit_cast(uint16_t, x);
                    w[j / 2] = j & 1 ? (w[j / 2] & 0xffffu) | y << 16 : (w[j / 2] & 0xffff0000u) | y;
                }
            }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // piece c; -infinity for what is not of the row, and for a NaN
    __device__ __forceinline__ uint4 load(int c) const
    {
        uint4 v = make_uint4(R::BARRED, R::BARRED, R::BARRED, R::BARRED);
        if (c > 0 && c < pieces - 1) v = base[c];
        else if (c == 0 || c == pieces - 1) v = edge[c != 0];
        if (nans) {
            uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < EACH; ++j)
                if (is_nan(R::get(w, j))) {
                    if constexpr (sizeof(E) == 4) w[j] = R::BARRED;
                    else w[j / 2] = j & 1 ? (w[j / 2] & 0xffffu) | (R::BARRED & 0xffff0000u) : (w[j / 2] & 0xffff0000u) | (R::BARRED & 0xffffu);
                }
            v = make_uint4(w[0], w[1], w[2], w[3]);
        }
        return v;
    }
    static __device__ __forceinline__ uint32_t key(const uint32_t *w, int j) { return key_of(R::get(w, j)); }
    __device__ __forceinline__ int index(int c, int j) const { return c * EACH - skip + j; }
    // f(number of the piece, piece) for all pieces of this wavefront, a lane's next SA_UNROLL being asked for meanwhile; done(step) after
    // each SA_UNROLL of them
    template <typename F, typename D>
    __device__ __forceinline__ void each(F f, D done) const
    {
        const int lane = threadIdx.x & 63, c0 = (threadIdx.x >> 6) * per, end = c0 + per < pieces ? c0 + per : pieces;
        uint4 v[SA_UNROLL];
#pragma unroll
        for (int i = 0; i < SA_UNROLL; ++i)
            if (c0 + i * HX_WAVE < end) v[i] = load(c0 + i * HX_WAVE + lane);
#pragma unroll 1
        for (int at = c0; at < c0 + per; at += SA_STEP) {
#pragma unroll
            for (int i = 0; i < SA_UNROLL; ++i)
                if (at + i * HX_WAVE < end) {
                    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                    f(at + i * HX_WAVE + lane, w);
                    if (at + SA_STEP + i * HX_WAVE < end) v[i] = load(at + SA_STEP + i * HX_WAVE + lane);
                }
            done((at - c0) / SA_STEP);
        }
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const { each(f, [](int) {}); }
};

__device__ __forceinline__ uint64_t wave_sum(uint64_t x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
// inclusive
__device__ __forceinline__ uint64_t wave_scan(uint64_t x)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < HX_WAVE; d <<= 1) {
        const uint64_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// What stays: elements before the last one, and that one.
struct Limit {
    uint32_t key;             // of the last that stays
    int idx;                  // its number: of equal keys those up to it stay
    __device__ __forceinline__ bool holds(uint32_t k, int i) const { return k > key || (k == key && i <= idx); }
};

// Weights of a row: 2^q exp((x - top) / T) = 2^q 2^(z / 32).  z's whole part picks a number of the table and the exponent, the rest,
// |f| <= 1/2, goes through the series of exp(f ln 2 / 32) up to f^5: 2^-48 of the weight.  Without branches, so that several elements' steps
// lie beside each other.
struct Weights {
    double top, inv;          // 32 log2(e) / T
    const double *tab;
    int q;
    bool boundless;           // the largest is +infinity, which takes all the weight: top 0 and inv 1, and all others as if -infinity
    uint32_t hi;

    // a logit as the functions below take it
    __device__ __forceinline__ float logit(float x) const { return boundless ? (x == __builtin_inff() ? 0.0f : -__builtin_inff()) : x; }
    // z; weights of 2^-1000 and less are one
    __device__ __forceinline__ double reach(float x) const { return fmax(((double)x - top) * inv, -32000.0); }
    __device__ __forceinline__ int bin(float x) const
    {
        const int b = -(int)__builtin_bit_cast(uint64_t, reach(x) + 6755399441055744.0);     // 1.5 2^52: the nearest whole number in the low bits
        return b < SA_BINS - 1 ? b : SA_BINS - 1;
    }
    __device__ __forceinline__ int bin(uint32_t k) const { return bin(logit(of_key(k))); }
    // the weight, and its bin
    __device__ __forceinline__ double scaled(uint32_t k, int *b) const { return scaled(logit(of_key(k)), b); }
    __device__ __forceinline__ double scaled(float x, int *b) const
    {
        const double z = reach(x), t = z + 6755399441055744.0, f = z - (t - 6755399441055744.0);
        const int n = (int)__builtin_bit_cast(uint64_t, t);
        double p = 3.9737099845494154e-11;                    // (ln 2 / 32)^5 / 5!
        p = __builtin_fma(p, f, 9.172562701824643e-09);
        p = __builtin_fma(p, f, 1.6938509724371819e-06);
        p = __builtin_fma(p, f, 2.3459619820224677e-04);
        p = __builtin_fma(p, f, 2.166084939249829e-02);
        p = __builtin_fma(p, f, 1.0);
        *b = -n < SA_BINS - 1 ? -n : SA_BINS - 1;
        // 2^(n / 32 + q): the exponent goes into the table's number
        const uint64_t power = __builtin_bit_cast(uint64_t, tab[n & 31]) + ((uint64_t)(uint32_t)((n >> 5) + q) << 52);
        return p * __builtin_bit_cast(double, power);
    }
    // to the nearest whole number; it is below 2^51
    static __device__ __forceinline__ uint64_t whole(double w) { return __builtin_bit_cast(uint64_t, w + 4503599627370496.0) & 0xfffffffffffffull; }
    __device__ __forceinline__ uint64_t mass(uint32_t k) const { int b; return whole(scaled(k, &b)); }
};

// Which elements a limit leaves, by one comparison each: up to the limit's piece those from its logit on, after it those beyond.  Only the
// piece itself is looked at number by number, and all of them where the limit is +infinity, as no number lies beyond it.
template <typename E>
struct Cut {
    Limit lim;
    float from, beyond;
    int piece;
    __device__ __forceinline__ Cut(const Row<E> &row, const Limit &l)
        : lim(l), from(of_key(l.key)), beyond(of_key(l.key < KEY_INF ? l.key + 1 : l.key)), piece(l.idx == 0x7fffffff ? l.idx : (l.idx + row.skip) / Row<E>::EACH) {}
    // a piece's logits, -infinity for what does not stay; whether any of the wavefront's does
    __device__ __forceinline__ bool stay(const Row<E> &row, const Weights &wt, int c, const uint32_t *p, float *x, bool *held) const
    {
        const float least = c <= piece ? from : beyond;
        bool some = false;
#pragma unroll
        for (int j = 0; j < Row<E>::EACH; ++j) {
            x[j] = Row<E>::R::get(p, j);
            held[j] = x[j] >= least;
        }
        if (lim.key >= KEY_INF || __builtin_amdgcn_ballot_w64(c == piece))
#pragma unroll
            for (int j = 0; j < Row<E>::EACH; ++j) held[j] = lim.holds(row.key(p, j), row.index(c, j));
#pragma unroll
        for (int j = 0; j < Row<E>::EACH; ++j) {
            some |= held[j];
            x[j] = held[j] ? x[j] : -__builtin_inff();
        }
        if (wt.boundless)
#pragma unroll
            for (int j = 0; j < Row<E>::EACH; ++j) x[j] = wt.logit(x[j]);
        return __builtin_amdgcn_ballot_w64(some);
    }
};

// The lowest element at which the sum of their masses in the order of the numbers exceeds target(total); -1: nowhere.  masses(number of the
// piece, piece, out) gives those of a piece's elements and returns how many of them count; *count = how many do in all.
template <typename E, typename M, typename W>
__device__ __forceinline__ int locate(const Row<E> &row, Shared &s, M masses, W target, uint64_t *total, int *count)
{
    constexpr int EACH = Row<E>::EACH;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, steps = row.per / SA_STEP;
    int mine = 0;
    uint64_t x = 0;
    __syncthreads();
    row.each([&](int c, const uint32_t *p) {
        uint64_t q[EACH];
        mine += masses(c, p, q);
#pragma unroll
        for (int j = 0; j < EACH; ++j) x += q[j];
    }, [&](int step) {
        x = wave_sum(x);
        if (lane == 0) s.hist[w * steps + step] = x;
        x = 0;
    });
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) mine += __shfl_xor(mine, d);
    if (lane == 0) s.wmin[w] = mine;
    if (tid == 0) s.r32[0] = -1;
    __syncthreads();
    // the step at which it is exceeded, and the element: the first wavefront
    if (w == 0) {
        uint64_t all = 0;
        for (int i = lane; i < SA_WAVES * steps; i += HX_WAVE) all += s.hist[i];
        all = wave_sum(all);
        const uint64_t want = target(all);
        uint64_t before = 0;
        int at = -1;
        for (int i0 = 0; i0 < SA_WAVES * steps && at < 0; i0 += HX_WAVE) {
            const uint64_t y = i0 + lane < SA_WAVES * steps ? s.hist[i0 + lane] : 0, sum = wave_scan(y);
            const unsigned long long m = __builtin_amdgcn_ballot_w64(before + sum > want);
            if (m) {
                const int l = __builtin_ctzll(m);
                at = i0 + l;
                before += __shfl(sum - y, l);
            } else before += __shfl(sum, 63);
        }
        if (lane == 0) {
            s.r32[1] = at;
            s.r64[0] = all;
            s.r64[1] = want - before;
        }
    }
    __syncthreads();
    // the pieces of that step: a wavefront each
    const int at = s.r32[1];
    const uint64_t want = s.r64[1];
    uint64_t q[EACH], sum = 0, own = 0;
    const int c = at < 0 ? 0 : (at / steps) * row.per + (at % steps) * SA_STEP + w * HX_WAVE + lane;
    if (at >= 0 && w < SA_UNROLL) {
        const uint4 v = row.load(c);
        const uint32_t p[4] = {v.x, v.y, v.z, v.w};
        (void)masses(c, p, q);
#pragma unroll
        for (int j = 0; j < EACH; ++j) own += q[j];
        sum = wave_scan(own);
        if (lane == 63) s.wave[w] = sum;
    }
    __syncthreads();
    if (at >= 0 && w < SA_UNROLL) {
        uint64_t run = sum - own;
        for (int i = 0; i < w; ++i) run += s.wave[i];
        if (run <= want && want < run + own)
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                if (run <= want && want < run + q[j]) s.r32[0] = row.index(c, j);
                run += q[j];
            }
    }
    __syncthreads();
    const int got = s.r32[0];
    *total = s.r64[0];
    int n = 0;
    for (int i = 0; i < SA_WAVES; ++i) n += s.wmin[i];
    *count = n;
    __syncthreads();
    return got;
}

// Of sums in order, EACH of a thread's beside each other, the one at which the whole exceeds or reaches `limit`: b < limit <= b + x.
// Its number in s.r32[1] (-1: none), what is before it in s.r64[0].  want(total) gives the limit the first time.
template <int EACH, typename W>
__device__ __forceinline__ void crossing(Shared &s, const uint64_t *x, uint64_t before, uint64_t *limit, bool first, W want)
{
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    uint64_t own = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) own += x[i];
    const uint64_t sum = wave_scan(own);
    if (lane == 63) s.wave[w] = sum;
    if (tid == 0) s.r32[1] = -1;
    __syncthreads();
    uint64_t b = before + sum - own, all = 0;
#pragma unroll
    for (int i = 0; i < SA_WAVES; ++i) {
        b += i < w ? s.wave[i] : 0;
        all += s.wave[i];
    }
    if (first) *limit = want(all);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (b < *limit && *limit <= b + x[i]) { s.r32[1] = tid * EACH + i; s.r64[0] = b; }
        b += x[i];
    }
    __syncthreads();
}

// The lowest key of lo .. hi for which f holds, which holds for all keys above one for which it does; hi if for none.  By 64 at a time.
template <typename F>
__device__ __forceinline__ uint32_t first_where(uint32_t lo, uint32_t hi, F f)
{
    while (lo < hi) {
        const uint32_t step = (hi - lo) / HX_WAVE + 1;
        const uint64_t at = (uint64_t)lo + (uint64_t)(threadIdx.x & 63) * step;
        const unsigned long long m = __builtin_amdgcn_ballot_w64(at >= hi || f((uint32_t)at));
        const int l = m ? __builtin_ctzll(m) : HX_WAVE;
        const uint64_t end = (uint64_t)lo + (uint64_t)l * step;
        if (l > 0) lo = (uint32_t)(end - step) + 1;
        hi = l == 0 ? lo : end < hi ? (uint32_t)end : hi;
    }
    return lo;
}

// The last element that stays of those for which `in` holds, in the order (logit falling, number rising): the one at which the sum of
// their weights (count_them: their number) reaches want(total).  EQUALS: the first *stay of those with the key are the last ones that stay.
enum Found { ALL_STAY, LAST_FOUND, EQUALS };
template <typename E, typename W>
__device__ __forceinline__ Found find_limit(const Row<E> &row, Shared &s, const Weights &wt, bool count_them, const Limit in, W want, Limit *out, uint64_t *stay)
{
    constexpr int EACH = Row<E>::EACH;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    auto mass = [&](uint32_t k) -> uint64_t { return count_them ? 1 : wt.mass(k); };
    uint32_t k_low = KEY_BARRED + 1, k_high = 0xffffffffu;       // keys still in question
    int shift = -1;                                              // -1: the weights' bins; else bins of (k_high - key) >> shift
    uint64_t before = 0, limit = 0;
    for (bool first = true;; first = false) {
        __syncthreads();
        for (int i = tid; i < SA_BINS * SA_COLS; i += SA_THREADS) s.hist[i] = 0;
        if (tid == 0) s.r32[2] = 0;
        __syncthreads();
        const Cut<E> cut(row, in);
        if (shift < 0 && count_them)
            row.each([&](int c, const uint32_t *p) {
                float x[EACH];
                bool held[EACH];
                if (!cut.stay(row, wt, c, p, x, held)) return;
                int b[EACH];
#pragma unroll
                for (int j = 0; j < EACH; ++j) b[j] = wt.bin(x[j]);
#pragma unroll
                for (int j = 0; j < EACH; ++j)
                    if (held[j]) atomicAdd((unsigned long long *)&s.hist[b[j] * SA_COLS + (lane & (SA_COLS - 1))], 1ull);
            });
        else if (shift < 0)
            row.each([&](int c, const uint32_t *p) {
                float x[EACH];
                bool held[EACH];
                if (!cut.stay(row, wt, c, p, x, held)) return;
                int b[EACH];
                uint64_t m[EACH];
#pragma unroll
                for (int j = 0; j < EACH; ++j) m[j] = Weights::whole(wt.scaled(x[j], &b[j]));
#pragma unroll
                for (int j = 0; j < EACH; ++j)
                    if (m[j]) atomicAdd((unsigned long long *)&s.hist[b[j] * SA_COLS + (lane & (SA_COLS - 1))], (unsigned long long)m[j]);
            });
        else row.each([&](int c, const uint32_t *p) {
            bool mine[EACH], some = false;
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const uint32_t k = row.key(p, j);
                mine[j] = k >= k_low && k <= k_high && in.holds(k, row.index(c, j));
                some |= mine[j];
            }
            if (!__builtin_amdgcn_ballot_w64(some)) return;
#pragma unroll
            for (int j = 0; j < EACH; ++j)
                if (mine[j]) {
                    const uint32_t k = row.key(p, j);
                    const uint64_t m = mass(k);
                    if (m) atomicAdd((unsigned long long *)&s.hist[((k_high - k) >> shift) * SA_COLS + (lane & (SA_COLS - 1))], (unsigned long long)m);
                }
        });
        __syncthreads();
        {
            uint64_t x[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (2 * tid + i < SA_BINS)
#pragma unroll
                    for (int j = 0; j < SA_COLS; ++j) x[i] += s.hist[(2 * tid + i) * SA_COLS + j];
            crossing<2>(s, x, before, &limit, first, want);
        }
        const int bin = s.r32[1];
        if (bin < 0) return ALL_STAY;
        before = s.r64[0];
        // the elements of that bin: their keys lie beside each other
        uint32_t first_key, last_key;
        if (shift >= 0) {
            const uint64_t below = (uint64_t)(bin + 1) << shift;
            last_key = k_high - ((uint32_t)bin << shift);
            first_key = k_high - k_low >= below ? k_high - (uint32_t)below + 1 : k_low;
        } else {
            const uint32_t most = k_high < wt.hi ? k_high : wt.hi;
            first_key = first_where(k_low, most, [&](uint32_t k) { return wt.bin(k) <= bin; });
            last_key = first_where(first_key, most, [&](uint32_t k) { return wt.bin(k) < bin; });
            if (wt.bin(last_key) < bin) --last_key;                 // (else none is nearer the top)
        }
        uint32_t lo = 0xffffffffu, hi = 0;
        row.each([&](int c, const uint32_t *p) {
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const uint32_t k = row.key(p, j);
                if (k >= first_key && k <= last_key && in.holds(k, row.index(c, j))) {
                    lo = k < lo ? k : lo;
                    hi = k > hi ? k : hi;
                    const int at = atomicAdd(&s.r32[2], 1);
                    if (at < SA_LIST) { s.lkey[at] = k; s.lidx[at] = row.index(c, j); }
                }
            }
        });
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const uint32_t a = __shfl_xor(lo, d), b = __shfl_xor(hi, d);
            lo = a < lo ? a : lo;
            hi = b > hi ? b : hi;
        }
        if (lane == 0) { s.wmin[w] = (int)lo; s.wmax[w] = (int)hi; }
        __syncthreads();
        int count = s.r32[2];
        for (int i = 0; i < SA_WAVES; ++i) {
            lo = (uint32_t)s.wmin[i] < lo ? (uint32_t)s.wmin[i] : lo;
            hi = (uint32_t)s.wmax[i] > hi ? (uint32_t)s.wmax[i] : hi;
        }
        if (count <= SA_LIST) {
            // in finer and finer bins until few are left of the list
            const int n = count;
            while (count > SA_FEW && lo != hi) {
                int sh = 0;
                while (((hi - lo) >> sh) >= SA_THREADS) ++sh;
                __syncthreads();
                s.hist[tid] = 0;
                if (tid == 0) s.r32[2] = 0;
                __syncthreads();
                for (int i = tid; i < n; i += SA_THREADS) {
                    const uint32_t k = s.lkey[i];
                    if (k >= lo && k <= hi) atomicAdd((unsigned long long *)&s.hist[(hi - k) >> sh], (unsigned long long)mass(k));
                }
                __syncthreads();
                const uint64_t x[1] = {s.hist[tid]};
                crossing<1>(s, x, before, &limit, false, want);
                const int b = s.r32[1];
                before = s.r64[0];
                const uint32_t top = hi - ((uint32_t)b << sh);
                const uint64_t floor_ = (uint64_t)((uint32_t)b + 1) << sh;         // of hi - key in the bins up to this one
                lo = hi - lo >= floor_ ? hi - (uint32_t)floor_ + 1 : lo;
                hi = top;
                int mine = 0;
                for (int i = tid; i < n; i += SA_THREADS) mine += s.lkey[i] >= lo && s.lkey[i] <= hi;
#pragma unroll
                for (int d = 32; d > 0; d >>= 1) mine += __shfl_xor(mine, d);
                if (lane == 0 && mine) atomicAdd(&s.r32[2], mine);
                __syncthreads();
                count = s.r32[2];
            }
            if (count <= SA_FEW) {
                __syncthreads();
                if (tid == 0) s.r32[2] = 0;
                __syncthreads();
                uint4 *few = (uint4 *)s.hist;
                for (int i = tid; i < n; i += SA_THREADS) {
                    const uint32_t k = s.lkey[i];
                    if (k >= lo && k <= hi) {
                        const uint64_t x = mass(k);
                        few[atomicAdd(&s.r32[2], 1)] = make_uint4(k, (uint32_t)s.lidx[i], (uint32_t)x, (uint32_t)(x >> 32));
                    }
                }
                __syncthreads();
                if (tid < count) {
                    const uint4 own = few[tid];
                    const uint64_t x = (uint64_t)own.w << 32 | own.z;
                    uint64_t b = before;
#pragma unroll 8
                    for (int j = 0; j < count; ++j) {
                        const uint4 o = few[j];
                        b += o.x > own.x || (o.x == own.x && (int)o.y < (int)own.y) ? (uint64_t)o.w << 32 | o.z : 0;
                    }
                    if (b < limit && limit <= b + x) { s.r32[3] = (int)own.y; s.r64[1] = own.x; }
                }
                __syncthreads();
                out->key = (uint32_t)s.r64[1];
                out->idx = s.r32[3];
                __syncthreads();
                return LAST_FOUND;
            }
        }
        if (lo == hi) {
            const uint64_t x = mass(lo);
            *stay = (limit - before + x - 1) / x;
            out->key = lo;
            return EQUALS;
        }
        k_low = lo;
        k_high = hi;
        shift = 0;
        while (((hi - lo) >> shift) >= SA_BINS) ++shift;
    }
}

struct Settings {
    int k;
    float p, u;
    double min_w;
};

// Sum over the workgroup's threads.
__device__ __forceinline__ uint64_t block_sum(Shared &s, uint64_t x)
{
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.wave[threadIdx.x >> 6] = x;
    __syncthreads();
    uint64_t all = 0;
#pragma unroll
    for (int i = 0; i < SA_WAVES; ++i) all += s.wave[i];
    return all;
}

// The rest of the way where only the elements with keys from `least` on can stay and they are few: an element a thread, each compared with
// all others.  False: they are more.
template <typename E>
__device__ __forceinline__ bool finish_short(const Row<E> &row, Shared &s, const Weights &wt, const Settings &g, uint32_t least, int *token, int *kept, uint64_t *total)
{
    const int tid = threadIdx.x;
    __syncthreads();
    if (tid == 0) s.r32[2] = 0;
    __syncthreads();
    row.each([&](int c, const uint32_t *p) {
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < Row<E>::EACH; ++j) {
            const uint32_t k = row.key(p, j);
            most = k > most ? k : most;
        }
        if (!__builtin_amdgcn_ballot_w64(most >= least)) return;
#pragma unroll
        for (int j = 0; j < Row<E>::EACH; ++j) {
            const uint32_t k = row.key(p, j);
            if (k >= least) {
                const int at = atomicAdd(&s.r32[2], 1);
                if (at < SA_SHORT) { s.lkey[at] = k; s.lidx[at] = row.index(c, j); }
            }
        }
    });
    __syncthreads();
    const int n = s.r32[2];
    if (n > SA_SHORT) return false;
    const bool mine = tid < n;
    const uint32_t k = mine ? s.lkey[tid] : wt.hi;
    const int idx = mine ? s.lidx[tid] : 0;
    int b;
    const double y = wt.scaled(k, &b);
    uint64_t x = mine ? Weights::whole(y) : 0;
    uint4 *all = (uint4 *)s.hist;
    if (tid < SA_SHORT) all[tid] = make_uint4(k, (uint32_t)idx, (uint32_t)x, (uint32_t)(x >> 32));
    __syncthreads();
    int rank = 0;
    uint64_t before = 0;
    if (mine)
#pragma unroll 8
        for (int j = 0; j < n; ++j) {
            const uint4 o = all[j];
            const bool earlier = o.x > k || (o.x == k && (int)o.y < idx);
            rank += earlier;
            before += earlier ? (uint64_t)o.w << 32 | o.z : 0;
        }
    bool stays = mine && (g.k <= 0 || rank < g.k);
    if (g.p < 1.0f) {
        uint64_t limit = 1;
        const uint64_t sum = block_sum(s, stays ? x : 0);
        if (g.p > 0.0f) {
            bool rest;
            limit = scaled(g.p, sum, &rest) + rest;
            limit = limit ? limit : 1;
        }
        stays = stays && before < limit;
    }
    stays = stays && y >= g.min_w;
    x = stays ? x : 0;
    *total = block_sum(s, x);
    if (tid < SA_SHORT) { all[tid].z = (uint32_t)x; all[tid].w = (uint32_t)(x >> 32); }
    *kept = (int)block_sum(s, stays);
    bool rest;
    const uint64_t want = scaled(g.u, *total, &rest);
    before = 0;
    if (mine)
#pragma unroll 8
        for (int j = 0; j < n; ++j) {
            const uint4 o = all[j];
            before += (int)o.y < idx ? (uint64_t)o.w << 32 | o.z : 0;
        }
    if (stays && before <= want && want < before + x) s.r32[0] = idx;
    __syncthreads();
    *token = s.r32[0];
    return true;
}

template <typename E>
__global__ __launch_bounds__(SA_THREADS) void hx_sample_kernel(SampleArgs a)
{
    using R = Raw<E>;
    __shared__ Shared s;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    Row<E> row;
    row.set((const E *)a.logits + (int64_t)r * a.row_stride, a.n_vocab, s.edge);

    const float T = a.temperature ? a.temperature[r] : 1.0f, p = a.top_p ? a.top_p[r] : 1.0f, mp = a.min_p ? a.min_p[r] : 0.0f, u = a.u[r];
    const int k = a.top_k ? a.top_k[r] : 0;
    const bool fine = !is_nan(T) && !is_nan(p) && !is_nan(mp) && !is_nan(u) && T >= 0.0f && __float_as_uint(T) != 0x7f800000u && mp >= 0.0f && mp <= 1.0f &&
                      u >= 0.0f && u < 1.0f;
    if (tid < 32) s.tab[tid] = exp2((double)tid / 32.0);

    // the largest logit; a NaN of either sign lies beyond the infinities in the order of the bits
    constexpr bool WIDE = sizeof(E) == 4;
    int hi = WIDE ? (int)0x80000000 : (int)0x80008000, lo = WIDE ? 0x7fffffff : 0x7fff7fff;
    row.each([&](int, const uint32_t *piece) { R::extremes(piece, hi, lo); });
    if constexpr (!WIDE) {
        const int h0 = (short)hi, h1 = hi >> 16, l0 = (short)lo, l1 = lo >> 16;
        hi = h0 > h1 ? h0 : h1;
        lo = l0 < l1 ? l0 : l1;
    }
    const int own_hi = hi;
    auto over_all = [&](int &most, int &least) {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const int x = __shfl_xor(most, d), y = __shfl_xor(least, d);
            most = x > most ? x : most;
            least = y < least ? y : least;
        }
        __syncthreads();
        if (lane == 0) { s.wmax[w] = most; s.wmin[w] = least; }
        __syncthreads();
        for (int i = 0; i < SA_WAVES; ++i) {
            most = s.wmax[i] > most ? s.wmax[i] : most;
            least = s.wmin[i] < least ? s.wmin[i] : least;
        }
    };
    over_all(hi, lo);
    uint32_t top_key;
    if (hi > R::INF || lo < ~R::INF) {
        row.nans = true;
        if (tid == 0) hx_raise(a.status, HX_ERR_INVALID_ARG);
        int most = 0, least = 0;                             // of the keys, shifted into the signed range
        row.each([&](int, const uint32_t *piece) {
#pragma unroll
            for (int j = 0; j < R::EACH; ++j) {
                const int x = (int)(row.key(piece, j) >> 1);
                most = x > most ? x : most;
            }
        });
        over_all(most, least);
        // the last bit is lost: it is the same for all but full-precision logits, where it is looked for
        uint32_t best = 0;
        row.each([&](int, const uint32_t *piece) {
#pragma unroll
            for (int j = 0; j < R::EACH; ++j) {
                const uint32_t x = row.key(piece, j);
                if ((int)(x >> 1) == most && x > best) best = x;
            }
        });
        int odd = (int)(best & 1);
        if (best == 0) odd = 0;
        least = 0;
        over_all(odd, least);
        top_key = (uint32_t)most << 1 | (uint32_t)odd;
    } else top_key = key_of(R::of_order(hi));
    __syncthreads();
    if (!fine && tid == 0) hx_raise(a.status, HX_ERR_INVALID_ARG);
    if (!fine || top_key <= KEY_BARRED) {
        if (tid == 0) {
            a.token[r] = -1;
            if (a.logprob) a.logprob[r] = -__builtin_inff();
            if (a.n_kept) a.n_kept[r] = 0;
        }
        return;
    }
    const bool boundless = top_key == KEY_INF;
    const Weights wt{boundless ? 0.0 : (double)of_key(top_key), boundless ? 1.0 : 46.16624130844683 / (double)T, s.tab, a.qbits, boundless, top_key};
    const double min_w = __builtin_ldexp((double)mp, a.qbits);
    Limit lim{KEY_BARRED + 1, 0x7fffffff};                 // all that are not barred
    uint64_t all;
    int kept, t = -1;
    auto answer = [&] {
        if (tid != 0) return;
        a.token[r] = t;
        if (a.n_kept) a.n_kept[r] = kept;
        if (a.logprob) {
            const double d = wt.boundless ? 0.0 : ((double)to_float(row.p[t]) - wt.top) / (double)T;
            a.logprob[r] = (float)(d - (log((double)all) - a.qbits * 0.6931471805599453));
        }
    };
    // Where few elements can stay, a key below which none does, and those from it on alone.  top-k: 1024 threads have each seen the largest
    // of their part; none of the first k of all is below the k-th of these, and not many others are above it (k = 320: 383 are expected).  min-p alone: its weight, and
    // 1 / 32 of a power of 2 less.
    if (T != 0.0f && ((k > 0 && k < a.n_vocab && k <= SA_SHORT * 5 / 8 && !row.nans) || (k <= 0 && p >= 1.0f && mp > 0.0f))) {
        uint32_t least = 0;
        if (k > 0) {
            const uint32_t own = key_of(R::of_order(own_hi));
            for (int i = tid; i < SA_BINS * SA_COLS; i += SA_THREADS) s.hist[i] = 0;
            __syncthreads();
            const bool some = own > KEY_BARRED && own <= top_key;          // the thread has an element that is not barred
            const int b = some ? wt.bin(own) : 0;
            if (some) atomicAdd((unsigned long long *)&s.hist[b * SA_COLS + (lane & (SA_COLS - 1))], 1ull);
            __syncthreads();
            uint64_t x[2] = {0, 0}, limit = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (2 * tid + i < SA_BINS)
#pragma unroll
                    for (int j = 0; j < SA_COLS; ++j) x[i] += s.hist[(2 * tid + i) * SA_COLS + j];
            crossing<2>(s, x, 0, &limit, true, [&](uint64_t) { return (uint64_t)k; });
            const int bin = s.r32[1];
            if (bin >= 0) {
                uint32_t mine = some && b <= bin ? own : 0xffffffffu;
#pragma unroll
                for (int d = 32; d > 0; d >>= 1) {
                    const uint32_t x2 = __shfl_xor(mine, d);
                    mine = x2 < mine ? x2 : mine;
                }
                if (lane == 0) s.wmin[w] = (int)mine;
                __syncthreads();
                least = 0xffffffffu;
                for (int i = 0; i < SA_WAVES; ++i) least = (uint32_t)s.wmin[i] < least ? (uint32_t)s.wmin[i] : least;
            }
        } else {
            const int bin = (int)(-32.0 * log2((double)mp)) + 2;
            if (bin < SA_BINS - 1) least = first_where(KEY_BARRED + 1, top_key, [&](uint32_t kk) { return wt.bin(kk) <= bin; });
        }
        if (least && finish_short(row, s, wt, {k, p, u, min_w}, least, &t, &kept, &all)) {
            answer();
            return;
        }
    }
    enum { TOP_K, TOP_P, TOKEN };
    // the least logit that min-p leaves
    const uint32_t least_mp = mp > 0.0f && T != 0.0f ? first_where(KEY_BARRED + 1, top_key, [&](uint32_t kk) { int b; return wt.scaled(kk, &b) >= min_w; }) : 0;
    for (int step = T == 0.0f ? TOKEN : TOP_K;; ++step) {
        // equal_key: elements of this key count 1 and no others; else the weights of all that stay
        bool equal = step == TOKEN && T == 0.0f;
        uint32_t equal_key = top_key;
        uint64_t stay = 1;
        if (step != TOKEN) {
            if (step == TOP_K ? k <= 0 || k >= a.n_vocab : p >= 1.0f) continue;
            const bool count_them = step == TOP_K;
            const Found found = find_limit(row, s, wt, count_them, lim, [&](uint64_t n) -> uint64_t {
                if (count_them) return (uint64_t)k < n ? (uint64_t)k : ~0ull;
                if (p <= 0.0f) return 1;
                bool rest;
                const uint64_t x = scaled(p, n, &rest) + rest;           // rounded up
                return x ? x : 1;
            }, &lim, &stay);
            if (found != EQUALS) continue;
            equal = true;
            equal_key = lim.key;
        }
        if (step == TOKEN && least_mp > lim.key) lim = {least_mp, 0x7fffffff};
        const Cut<E> cut(row, lim);
        t = locate(row, s, [&](int c, const uint32_t *piece, uint64_t *q) -> int {
            constexpr int EACH = R::EACH;
            int count = 0;
#pragma unroll
            for (int j = 0; j < EACH; ++j) q[j] = 0;
            if (equal) {
#pragma unroll
                for (int j = 0; j < EACH; ++j) { q[j] = row.key(piece, j) == equal_key; count += (int)q[j]; }
                return count;
            }
            float x[EACH];
            bool held[EACH];
            if (!cut.stay(row, wt, c, piece, x, held)) return 0;
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                int b;
                q[j] = Weights::whole(wt.scaled(x[j], &b));
                count += held[j];
            }
            return count;
        }, [&](uint64_t n) -> uint64_t {
            if (equal) return stay - 1;
            bool rest;
            return scaled(u, n, &rest);
        }, &all, &kept);
        if (step == TOKEN) break;
        lim.idx = t;
    }
    if (T == 0.0f) {
        if (tid == 0) {
            a.token[r] = t;
            if (a.logprob) a.logprob[r] = 0.0f;
            if (a.n_kept) a.n_kept[r] = 1;
        }
        return;
    }
    answer();
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
    HX_REQUIRE(ctx, n_rows <= hx_most_groups(SA_THREADS), HX_ERR_SHAPE, "%d rows in one call", n_rows);
    HxDeviceGuard guard(ctx->device);
    HX_REQUIRE(ctx, guard.ok, HX_ERR_DEVICE, "cannot select device %d", ctx->device);
    hipStream_t stream = (hipStream_t)stream_;
    int bits = 0;
    while (((int64_t)1 << bits) < n_vocab) ++bits;
    const int q = 61 - bits < 50 ? 61 - bits : 50;
    SampleArgs a{n_rows, n_vocab, q, logits, row_stride, temperature, top_k, top_p, min_p, u, token, logprob, n_kept, ctx->d_status};
    if (dtype == HX_F32) hx_sample_kernel<float><<<n_rows, SA_THREADS, 0, stream>>>(a);
    else if (dtype == HX_BF16) hx_sample_kernel<__bf16><<<n_rows, SA_THREADS, 0, stream>>>(a);
    else hx_sample_kernel<_Float16><<<n_rows, SA_THREADS, 0, stream>>>(a);
    return hx_check_launch(ctx, "hx_sample_kernel");
}
