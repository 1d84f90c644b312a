// The n-th largest of many keys, by a workgroup.
#pragma once

#include "hx_common.hpp"

namespace {

constexpr int NTH_BINS = 1024, NTH_LIST = 64;

template <typename K, int THREADS>
struct NthState {
    static constexpr int WAVES = THREADS / HX_WAVE;
    int bins[NTH_BINS];
    K list[NTH_LIST];
    K least[WAVES], most[WAVES];
    int count[WAVES];
    int above, n_list, bin;
    // found
    K edge;
    int equals;
};

template <typename K> __device__ __forceinline__ K nth_across(K x, int d)
{
    if constexpr (sizeof(K) == 8) return (K)__shfl_xor((uint32_t)((uint64_t)x >> 32), d) << 32 | __shfl_xor((uint32_t)x, d);
    else return __shfl_xor(x, d);
}

// s.edge = the n-th largest (n > 0) of key(from) .. key(to - 1), s.equals = how many equal to it are among the first n; s.edge = 0 where there are no more than n.
// Keys are whole numbers without a sign; those of 0 count for nothing.  They are dealt into bins of equal width between the least and the
// largest of those that are left, and the bin that holds the n-th is looked at again, until few enough are left to compare each with each: the
// least and the largest lie in different bins, so fewer are left each time.
template <typename K, int THREADS, typename F>
__device__ __forceinline__ void nth_largest(F key, int from, int to, int n, NthState<K, THREADS> &s)
{
    constexpr int WAVES = THREADS / HX_WAVE;
    const int tid = threadIdx.x, lane = tid & (HX_WAVE - 1), wave = tid / HX_WAVE;
    K lo = 1, hi = ~(K)0;                                   // those that are left
    for (bool first = true;; first = false) {
        K least = ~(K)0, most = 0;
        int left = 0;
        for (int i = from + tid; i < to; i += THREADS) {
            const K x = key(i);
            if (x < lo || x > hi) continue;
            ++left;
            least = x < least ? x : least;
            most = x > most ? x : most;
        }
#pragma unroll
        for (int d = HX_WAVE / 2; d > 0; d >>= 1) {
            const K l = nth_across(least, d), m = nth_across(most, d);
            least = l < least ? l : least;
            most = m > most ? m : most;
            left += __shfl_xor(left, d);
        }
        __syncthreads();                                    // whoever still reads what is written now
        if (lane == 0) { s.least[wave] = least; s.most[wave] = most; s.count[wave] = left; }
        for (int i = tid; i < NTH_BINS; i += THREADS) s.bins[i] = 0;
        if (tid == 0) s.n_list = 0;
        __syncthreads();
        left = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            least = s.least[w] < least ? s.least[w] : least;
            most = s.most[w] > most ? s.most[w] : most;
            left += s.count[w];
        }
        if (left <= n || least == most) {
            if (tid == 0) {
                s.edge = left > n ? least : first ? 0 : least;
                s.equals = left > n ? n : INT32_MAX;
            }
            __syncthreads();
            return;
        }
        if (left <= NTH_LIST) {
            for (int i = from + tid; i < to; i += THREADS) {
                const K x = key(i);
                if (x >= least && x <= most) s.list[atomicAdd(&s.n_list, 1)] = x;
            }
            __syncthreads();
            for (int k = tid; k < left; k += THREADS) {
                const K x = s.list[k];
                int larger = 0, equal = 0;
                for (int i = 0; i < left; ++i) { larger += s.list[i] > x; equal += s.list[i] == x; }
                if (larger < n && larger + equal >= n) { s.edge = x; s.equals = n - larger; }          // (all that are equal write the same)
            }
            __syncthreads();
            return;
        }
        // bins of 2^shift
        int bits;
        if constexpr (sizeof(K) == 8) bits = 64 - __builtin_clzll(most - least);
        else bits = 32 - __builtin_clz(most - least);
        const int shift = bits > 10 ? bits - 10 : 0;
        static_assert(NTH_BINS == 1 << 10);
        for (int i = from + tid; i < to; i += THREADS) {
            const K x = key(i);
            if (x >= least && x <= most) atomicAdd(s.bins + (int)((x - least) >> shift), 1);
        }
        __syncthreads();
        if (wave == 0) {
            // a lane's bins, the highest first, and how many lie in those of the lanes before it
            constexpr int EACH = NTH_BINS / HX_WAVE;
            int mine = 0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) mine += s.bins[NTH_BINS - 1 - lane * EACH - i];
            int before = mine;
#pragma unroll
            for (int d = 1; d < HX_WAVE; d <<= 1) { const int y = __shfl_up(before, d); if (lane >= d) before += y; }
            before -= mine;
            if (before < n && before + mine >= n)
                for (int i = 0; i < EACH; ++i) {
                    const int at = NTH_BINS - 1 - lane * EACH - i, c = s.bins[at];
                    if (before + c >= n) { s.bin = at; s.above = before; break; }
                    before += c;
                }
        }
        __syncthreads();
        n -= s.above;
        lo = least + ((K)s.bin << shift);
        const K width = ((K)1 << shift) - 1;
        hi = most - lo < width ? most : lo + width;
    }
}

// The same of keys that the threads hold, EACH a thread (0: none): the range between the least and the largest is halved until as many lie above as are wanted,
// by counts of the wavefronts, which meet once for each halving.
template <typename K, int THREADS>
struct NthHeld {
    static constexpr int WAVES = THREADS / HX_WAVE;
    K least[WAVES], most[WAVES], last[WAVES];
    int count[2][WAVES];
};
template <typename K, int THREADS, int EACH>
__device__ __forceinline__ void nth_largest_held(const K (&x)[EACH], int n, NthHeld<K, THREADS> &s, K *edge, int *equals)
{
    constexpr int WAVES = THREADS / HX_WAVE;
    const int lane = threadIdx.x & (HX_WAVE - 1), wave = threadIdx.x / HX_WAVE;
    auto extreme = [](K a, K b, bool largest) { return (b > a) == largest ? b : a; };
    auto over_lanes = [&](K y, bool largest) {
#pragma unroll
        for (int d = HX_WAVE / 2; d > 0; d >>= 1) y = extreme(y, nth_across(y, d), largest);
        return y;
    };
    auto over_waves = [&](K y, K *to, bool largest) {
        if constexpr (WAVES > 1) {
            if (lane == 0) to[wave] = y;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) y = extreme(y, to[w], largest);
        }
        return y;
    };
    int turn = 0;
    auto at_least = [&](K y) {                              // how many keys are y or more
        int c = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) c += __builtin_popcountll(__builtin_amdgcn_ballot_w64(x[i] >= y));
        if constexpr (WAVES > 1) {
            if (lane == 0) s.count[turn][wave] = c;
            __syncthreads();
            c = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) c += s.count[turn][w];
            turn ^= 1;                                      // (who is still reading the other has passed a barrier since)
        }
        return c;
    };
    K least = ~(K)0, most = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        least = x[i] != 0 && x[i] < least ? x[i] : least;
        most = x[i] > most ? x[i] : most;
    }
    least = over_waves(over_lanes(least, false), s.least, false);
    most = over_waves(over_lanes(most, true), s.most, true);
    *edge = 0;
    *equals = INT32_MAX;
    if (at_least(1) <= n) return;
    // more than n keys are `least` or more, fewer than n are more than `most`
    while (least < most) {
        const K mid = most - (most - least) / 2;
        const int above = at_least(mid);
        if (above == n) {                                   // the least of them is the n-th
            K y = ~(K)0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) y = x[i] >= mid && x[i] < y ? x[i] : y;
            *edge = over_waves(over_lanes(y, false), s.last, false);
            return;
        }
        if (above > n) least = mid; else most = mid - 1;
    }
    *edge = least;
    *equals = n - (least == ~(K)0 ? 0 : at_least(least + 1));
}

// Order of a number that is no NaN, as a key: larger numbers have larger keys, -infinity has the least.
__device__ __forceinline__ uint64_t nth_key(double x)
{
    const int64_t v = __builtin_bit_cast(int64_t, x);
    return (uint64_t)(v ^ (v >> 63 | INT64_MIN));
}

}  // namespace
