// What the calls that take, give back and move pages share.
#pragma once

#include "hx_serve.hpp"

namespace {

constexpr int PL_THREADS = 1024;           // the planning workgroup
constexpr int PL_WAVES = PL_THREADS / HX_WAVE;

// Sum of x over the workgroup's threads before this one; *all = over all of them.  s: PL_WAVES words.
__device__ __forceinline__ int64_t block_before(int64_t x, int64_t *s, int64_t *all)
{
    const int lane = threadIdx.x & (HX_WAVE - 1), w = threadIdx.x / HX_WAVE;
    int64_t sum = x;
#pragma unroll
    for (int d = 1; d < HX_WAVE; d <<= 1) {
        const int64_t y = __shfl_up(sum, d);
        if (lane >= d) sum += y;
    }
    __syncthreads();
    if (lane == HX_WAVE - 1) s[w] = sum;
    __syncthreads();
    int64_t before = 0, total = 0;
#pragma unroll
    for (int i = 0; i < PL_WAVES; ++i) {
        const int64_t y = s[i];
        before += i < w ? y : 0;
        total += y;
    }
    *all = total;
    return before + sum - x;
}

// The first `want` pages that are free, ref <= 0 (USED: in use), from page `from` on and before `to`, into list; returns how many there are, at most `want`.
// A wavefront looks at 8 x 64 neighbouring pages at a time, the workgroup at 8192.
constexpr int SCAN_EACH = 8;
template <bool USED>
__device__ int first_pages(const int32_t *ref, int from, int to, int want, int32_t *list, int64_t *s)
{
    const int lane = threadIdx.x & (HX_WAVE - 1), w = threadIdx.x / HX_WAVE;
    int found = 0;
    for (int64_t at = from; at < to && found < want; at += PL_THREADS * SCAN_EACH) {
        const int64_t mine = at + w * (HX_WAVE * SCAN_EACH) + lane;
        int r[SCAN_EACH];
#pragma unroll
        for (int j = 0; j < SCAN_EACH; ++j) r[j] = mine + j * HX_WAVE < to ? ref[mine + j * HX_WAVE] : (USED ? 0 : 1);
        unsigned long long m[SCAN_EACH];
        int count = 0;
#pragma unroll
        for (int j = 0; j < SCAN_EACH; ++j) {
            m[j] = __builtin_amdgcn_ballot_w64((r[j] > 0) == USED);
            count += __builtin_popcountll(m[j]);
        }
        int64_t all;
        // every lane counts its wavefront's pages, lane 0's share is what is added up
        int64_t before = block_before(lane == 0 ? count : 0, s, &all);
        before = __shfl(before, 0);
        int rank = found + (int)before;
#pragma unroll
        for (int j = 0; j < SCAN_EACH; ++j) {
            const int mine_rank = rank + __builtin_popcountll(m[j] & ((1ull << lane) - 1));
            if (((m[j] >> lane) & 1) && mine_rank < want) list[mine_rank] = (int32_t)(mine + j * HX_WAVE);
            rank += __builtin_popcountll(m[j]);
        }
        found += (int)all;
    }
    __syncthreads();
    return found < want ? found : want;
}

// One of a pool's arrays, by a number that is the same for all threads.
struct Plane {
    char *at;
    int row_bytes;           // of a token in one head
};
__device__ __forceinline__ Plane plane(const KvPlanes &p, int i)
{
    return Plane{i == 0 ? p.at[0] : i == 1 ? p.at[1] : i == 2 ? p.at[2] : p.at[3], i < 2 ? p.row_bytes[0] : p.row_bytes[2]};
}

// f(U{}) with the widest type that rows of so many bytes consist of.  (An array of HIP's own uint4 that lives across a barrier goes to scratch memory.)
typedef uint32_t Four __attribute__((ext_vector_type(4)));
template <typename F>
__device__ __forceinline__ void by_width(int row_bytes, F f)
{
    if (row_bytes % 16 == 0) f(Four{});
    else if (row_bytes % 4 == 0) f(uint32_t{});
    else if (row_bytes % 2 == 0) f(uint16_t{});
    else f(uint8_t{});
}

// A page is held by one table less.  Counts that would go below 0 stay.
__device__ __forceinline__ void give_back(const KvView &kv, int page)
{
    if (page >= kv.n_pages) { hx_raise(kv.status, HX_ERR_INDEX); return; }
    if (atomicSub(kv.ref + page, 1) <= 0) { atomicAdd(kv.ref + page, 1); hx_raise(kv.status, HX_ERR_INDEX); }
}

}  // namespace
