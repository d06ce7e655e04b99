// Register-level pieces of the attention kernels.
#pragma once

#include "kv.h"
#include "kv_types.h"

namespace dro {

typedef Vec<float, 4> f32x4;
typedef Vec<float, 16> f32x16;
typedef Vec<uint32_t, 4> u32x4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Running maxima are raised only when a step exceeds them by 2^kSlack, so most steps
// rescale nothing; weights stay below 2^kSlack of that maximum's.  (With 0 a prompt of 8192 tokens,
// 64 heads on 8, takes 1136 us where 8 takes 1098.)
constexpr float kSlack = 8.0f;

// The running maximum m is held 2^kUnit below the largest score, so the largest weight of a row is
// 2^kUnit at least.  f16 weights are products' operands in f16, which ends at 2^-24: with a unit of
// 1 those below 2^-25 of the largest were lost, 1.4 % of the tail of 131,072 keys that lie 14.5
// below the first one's score.  With 2^7 the end is 2^-32 of the largest, and 2^(7 + kSlack) leaves
// an octave below f16's largest number.
template <class T> constexpr float kUnit = __is_same(T, f16) ? 7.0f : 0.0f;

// Whether a step of scores up to `mt` has to raise m.  f16: where the scores' last places are half
// an octave and more, always, so that the weights stay in range.
template <class T> __device__ __forceinline__ bool has_to_raise(float mt, float m)
{
    return mt > m + (kSlack + kUnit<T>) || (__is_same(T, f16) && fabsf(mt) >= 0x1p23f);
}

// 16 x 16 tile over 32 products.  First operand: lane holds row lane % 16, products
// (lane / 16) 8 .. + 8; second: column lane % 16, the same products; result: column
// lane % 16, rows (lane / 16) 4 .. + 4.
template <class T> __device__ __forceinline__ f32x4 mfma16(u32x4 x, u32x4 y, f32x4 c)
{
    if constexpr (__is_same(T, bf16))
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Vec<bf16, 8>, x),
                                                       __builtin_bit_cast(Vec<bf16, 8>, y), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Vec<f16, 8>, x),
                                                      __builtin_bit_cast(Vec<f16, 8>, y), c, 0, 0, 0);
}

template <class T> __device__ __forceinline__ uint32_t pack2(float x, float y)
{
    return __builtin_bit_cast(uint32_t, Vec<T, 2>{(T)x, (T)y});
}

// largest over the four groups of 16 lanes, lane by lane
__device__ __forceinline__ float max_groups(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    x = fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
    const uint32_t d = __builtin_bit_cast(uint32_t, x);
    r = __builtin_amdgcn_permlane16_swap(d, d, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float sum_groups(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    x = __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
    const uint32_t d = __builtin_bit_cast(uint32_t, x);
    r = __builtin_amdgcn_permlane16_swap(d, d, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// cap tanh(y) + add for x = 2 y log2 e, by tanh y = 1 - 2 / (2^x + 1): to 2^-21 of the cap
__device__ __forceinline__ float tanh_scaled(float x, float cap, float add)
{
    return __builtin_fmaf(-2.0f * cap, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x) + 1.0f), cap + add);
}

// the bits of the infinities and NaN among the values of a dword of the cache's type C: an
// exponent of ones (fp8: NaN alone) carries into the sign's place
template <class C> __device__ __forceinline__ uint32_t nonfinite_mask(uint32_t w)
{
    if constexpr (__is_same(C, fp8) || __is_same(C, mx8))
        return ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu;
    else if constexpr (__is_same(C, bf16))
        return ((((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu;
    else
        return ((((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u) >> 15) * 0xffffu;
}

// Whether the `bytes` (a multiple of 4) of a value row at `p` hold an infinity or a NaN; by a wave.
template <class C> __device__ __forceinline__ bool row_nonfinite(const char *p, int bytes)
{
    uint32_t bad = 0;
    for (int i = (threadIdx.x & 63) * 4; i < bytes; i += 256) bad |= nonfinite_mask<C>(*(const uint32_t *)(p + i));
    return __any(bad);
}

// The same of a row of codes in shared scales, as T: an infinity beyond f16's range, or a NaN.
template <class T, class C> __device__ __forceinline__ bool mx_row_nonfinite(const char *p, const uint8_t *powers, int D)
{
    bool bad = false;
    for (int d = threadIdx.x & 63; d < D; d += 64) bad |= !__builtin_isfinite(mx_value_at<T, C>(p, powers, d));
    return __any(bad);
}

// N dwords at base + off, aligned to 8 elements of the cache's type: the base is the same
// for the wave, so an address costs no 64-bit vector arithmetic.
template <int N> struct Words {
    uint32_t w[N];
};
template <int N> __device__ __forceinline__ Words<N> load_words(const char *base, uint32_t off)
{
    Words<N> x;
    if constexpr (N >= 4) {
        typedef u32x4 __attribute__((aligned(8))) loose;
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const u32x4 y = *(const loose *)(base + 16 * i + off);
#pragma unroll
            for (int j = 0; j < 4; ++j) x.w[4 * i + j] = y[j];
        }
    } else if constexpr (N == 2) {
        typedef Vec<uint32_t, 2> __attribute__((aligned(4))) loose;
        const Vec<uint32_t, 2> y = *(const loose *)(base + off);
        x.w[0] = y[0];
        x.w[1] = y[1];
    } else {
        x.w[0] = *(const uint32_t *)(base + off);
    }
    return x;
}

// The same of memory whose place is uniform but for a lane's offset and known in two parts: the
// address of a buffer (uniform, less than 2^31 bytes from its base on) stays in scalar registers, so
// that it takes one vector register whatever the row.  (Pointers: the compiler adds up a 64-bit
// vector address a load, and the loads on their way spill registers.)
struct Buffer {
    __amdgpu_buffer_rsrc_t r;
    // (the base: two words of an address)
    __device__ __forceinline__ Buffer(uint32_t low, uint32_t high)
        : r(__builtin_amdgcn_make_buffer_rsrc((void *)((uint64_t)high << 32 | low), 0, 0x7fffffff, 0x00020000))
    {
    }
    template <int N> __device__ __forceinline__ Words<N> words(uint32_t lane, uint32_t uniform) const
    {
        Words<N> x;
        if constexpr (N == 1) {
            x.w[0] = __builtin_amdgcn_raw_buffer_load_b32(r, lane, uniform, 0);
        } else if constexpr (N == 2) {
            const auto y = __builtin_amdgcn_raw_buffer_load_b64(r, lane, uniform, 0);
            x.w[0] = y[0];
            x.w[1] = y[1];
        } else {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                const auto y = __builtin_amdgcn_raw_buffer_load_b128(r, lane, uniform + 16 * i, 0);
#pragma unroll
                for (int j = 0; j < 4; ++j) x.w[4 * i + j] = y[j];
            }
        }
        return x;
    }
    __device__ __forceinline__ uint32_t half(uint32_t lane, uint32_t uniform) const
    {
        return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, lane, uniform, 0);
    }
    __device__ __forceinline__ uint32_t byte(uint32_t lane, uint32_t uniform) const
    {
        return (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r, lane, uniform, 0);
    }
};

// The rows of no request, by workgroup `nth` of `of`: those without other work, where there are
// any, since the others' way to their first keys is a chain of loads already.
template <class T> __device__ __forceinline__ void zero_rows(const KvAttnArgs &a, uint32_t nth, uint32_t of)
{
    const int t0 = min(max(a.start[0], 0), a.T), t1 = min(max(a.start[a.R], 0), a.T);
    const int lost = t0 + a.T - t1;
    for (uint32_t y = nth; y < (uint32_t)lost; y += of) {
        const int x = (int)y;
        const int t = x < t0 ? x : t1 + x - t0;
        for (int i = threadIdx.x; i < a.Hq * a.D; i += blockDim.x) {
            const int h = i / a.D;
            ((T *)a.out)[t * a.out_token + h * a.out_head + (i - h * a.D)] = (T)0.0f;
        }
        if (a.lse)
            for (int h = threadIdx.x; h < a.Hq; h += blockDim.x) a.lse[(int64_t)t * a.Hq + h] = -INFINITY;
    }
}

}  // namespace dro
