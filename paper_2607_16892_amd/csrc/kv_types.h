// Element types of the paged cache and their conversions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dro.h"

namespace dro {

typedef __bf16 bf16;
typedef _Float16 f16;
struct fp8 {  // e4m3 with one NaN and no infinity (largest finite value 448)
    uint8_t bits;
};

template <class T, int N> using Vec = T __attribute__((ext_vector_type(N)));

__device__ __forceinline__ float to_float(bf16 x) { return (float)x; }
__device__ __forceinline__ float to_float(f16 x) { return (float)x; }

// Four floats as fp8, rounded to nearest even; what is beyond +-448 becomes +-448,
// NaN stays NaN.
__device__ __forceinline__ uint32_t pack_fp8(const float *f)
{
    float g[4];
    for (int j = 0; j < 4; ++j) g[j] = f[j] != f[j] ? f[j] : fminf(fmaxf(f[j], -448.0f), 448.0f);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(g[0], g[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(g[2], g[3], w, true);
}

// Two fp8 values (the low or the high half of `w`) as packed T, exactly.
template <class T, bool kHigh> __device__ __forceinline__ uint32_t unpack_fp8(uint32_t w)
{
    if constexpr (__is_same(T, bf16))
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, kHigh));
    else
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, kHigh));
}

// component d of a value row of the cache
template <class C> __device__ __forceinline__ float value_at(const char *row, int d)
{
    if constexpr (sizeof(C) == 1) {
        const uint32_t w = ((const uint8_t *)row)[d];
        return __builtin_bit_cast(float, unpack_fp8<bf16, false>(w) << 16);
    } else {
        return to_float(((const C *)row)[d]);
    }
}

}  // namespace dro
