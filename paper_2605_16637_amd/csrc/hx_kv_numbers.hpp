// A cache's stored numbers, one by one.
#pragma once

#include "hx_serve.hpp"

#include <type_traits>

namespace {

struct E2m1 {};                                                                  // the type of a pool of 4 bits; that of 8 is uint8_t
constexpr int E2M1_LEAST = 127 - 23, E2M1_MOST = 127 + 13, E2M1_NAN = 255;       // bytes of its scales

// N stored numbers from number `at` of the pool on, times their scale; of 4 bits all under one.
template <typename S, int N>
__device__ __forceinline__ void stored(const void *pool, const uint8_t *exps, float scale, int64_t at, float *x)
{
    if constexpr (std::is_same_v<S, E2m1>) {
        static_assert(N % 8 == 0 && N <= E2M1_GROUP);
        struct alignas(N / 2) Words { uint32_t w[N / 8]; } e = *(const Words *)((const char *)pool + at / 2);
        const int byte = exps[at / E2M1_GROUP];
        const float unit = byte == E2M1_NAN ? __builtin_nanf("") : __uint_as_float((uint32_t)byte << 23);
        typedef float Two __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const Two y[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e.w[i], unit, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e.w[i], unit, 1),
                              __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e.w[i], unit, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(e.w[i], unit, 3)};
#pragma unroll
            for (int j = 0; j < 8; ++j) x[8 * i + j] = y[j / 2][j % 2];
        }
    } else if constexpr (sizeof(S) == 1) {
        struct alignas(N < 16 ? N : 16) Words { uint32_t w[N / 4]; } e = *(const Words *)((const char *)pool + at);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int w = e.w[i / 4];
            const float y = i % 4 == 0 ? __builtin_amdgcn_cvt_f32_fp8(w, 0) : i % 4 == 1 ? __builtin_amdgcn_cvt_f32_fp8(w, 1)
                          : i % 4 == 2 ? __builtin_amdgcn_cvt_f32_fp8(w, 2) : __builtin_amdgcn_cvt_f32_fp8(w, 3);
            x[i] = y * scale;
        }
    } else {
        struct alignas(N < 8 ? 2 * N : 16) Numbers { S x[N]; } e = *(const Numbers *)((const S *)pool + at);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (float)e.x[i];
    }
}

}  // namespace
