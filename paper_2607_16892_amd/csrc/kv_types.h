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
// Shared scales: kGroup components of a row share a power of two, 2^(byte - 127), and are 4-bit
// codes (0, .5, 1, 1.5, 2, 3, 4, 6 and a sign; the even component in a byte's low half) or fp8.
struct mx4 {
    uint8_t pair;
};
struct mx8 {
    uint8_t bits;
};
constexpr int kGroup = 32;
template <class C> constexpr bool kMx = __is_same(C, mx4) || __is_same(C, mx8);

// bytes of n components (mx4: n is even)
template <class C, class N> __host__ __device__ constexpr N bytes_of(N n)
{
    return __is_same(C, mx4) ? n / 2 : n * (N)sizeof(C);
}

// Bytes from a row of a block to component d of the row n further (n < 16): unsigned, as rows of 4-bit
// codes lie up to 2^28 components apart, whose bytes alone stay below 2^31.
template <class C> __host__ __device__ constexpr uint32_t row_bytes(int n, int64_t stride, int d)
{
    return bytes_of<C>((uint32_t)n * (uint32_t)stride + (uint32_t)d);
}

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

template <class C> struct MxFormat {
    static constexpr bool kFour = __is_same(C, mx4);
    static constexpr int kTop = kFour ? 2 : 8;                        // exponent of the largest code
    static constexpr uint32_t kAbove = kFour ? 0x600000 : 0x680000;   // fraction beyond which the power grows
    static constexpr int kLeast = kFour ? -125 : -117;                // smallest code normal in bf16
    template <class T> static constexpr int kMost = (__is_same(T, f16) ? 15 : 127) - kTop;  // largest finite in T
};

// Pair kPair of the components in a dword of codes of scale `s`, as packed T: exact in bf16 (in f16
// rounded, infinite beyond its range), NaN where the group's byte is 255.
__device__ __forceinline__ float group_scale(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }
template <class T, class C, int kPair> __device__ __forceinline__ uint32_t unpack_mx(uint32_t w, float s)
{
    if constexpr (__is_same(C, mx4)) {
        if constexpr (__is_same(T, bf16))
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, kPair));
        else
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, kPair));
    } else {
        if constexpr (__is_same(T, bf16))
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, kPair));
        else
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, kPair));
    }
}
// Eight components, in one dword of mx4 or two of mx8, as packed T.
template <class T, class C> __device__ __forceinline__ Vec<uint32_t, 4> unpack_mx8of(const uint32_t *w, float s)
{
    if constexpr (__is_same(C, mx4))
        return Vec<uint32_t, 4>{unpack_mx<T, C, 0>(w[0], s), unpack_mx<T, C, 1>(w[0], s), unpack_mx<T, C, 2>(w[0], s),
                                unpack_mx<T, C, 3>(w[0], s)};
    else
        return Vec<uint32_t, 4>{unpack_mx<T, C, 0>(w[0], s), unpack_mx<T, C, 1>(w[0], s), unpack_mx<T, C, 0>(w[1], s),
                                unpack_mx<T, C, 1>(w[1], s)};
}

// component d of a row of codes, as T
template <class T, class C> __device__ __forceinline__ float mx_value_at(const char *row, const uint8_t *powers, int d)
{
    const uint32_t w = ((const uint8_t *)row)[bytes_of<C>(d & ~1)] |
                       (__is_same(C, mx8) ? (uint32_t)((const uint8_t *)row)[d | 1] << 8 : 0u);
    const uint32_t pair = unpack_mx<T, C, 0>(w, group_scale(powers[d / kGroup]));
    return to_float(__builtin_bit_cast(T, (uint16_t)(pair >> (d & 1) * 16)));
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
