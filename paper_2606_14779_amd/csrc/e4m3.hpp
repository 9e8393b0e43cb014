// Elements of 8-bit pages: e4m3 (largest 448, no infinities) times a power of two that 32 elements share (gfx950).
//
// A power of two costs no precision against any other scale, as e4m3 is a floating format, and makes the way back to
// bf16 or f16 exact: one instruction for two elements, which takes the power in the exponent field of a float.  The
// exponents are kept where every element is a normal bf16 (e >= -117: 2^(-9 - 117) = 2^-126) or a multiple of f16's
// smallest step (e >= -15: 2^(-9 - 15) = 2^-24), and finite (240 * 2^e at the largest e).
#ifndef KVP_E4M3_HPP
#define KVP_E4M3_HPP

#include "wave.hpp"

namespace kvp {

template <class T> struct E4M3;
template <> struct E4M3<BF16> {
    static constexpr int32_t kLeast = -117, kMost = 120;
    // elements 2 i and 2 i + 1 of a word, i = 0 or 1
    static __device__ __forceinline__ uint32_t low(uint32_t w, float power)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, false));
    }
    static __device__ __forceinline__ uint32_t high(uint32_t w, float power)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, true));
    }
};
template <> struct E4M3<F16> {
    static constexpr int32_t kLeast = -15, kMost = 8;
    static __device__ __forceinline__ uint32_t low(uint32_t w, float power)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, power, false));
    }
    static __device__ __forceinline__ uint32_t high(uint32_t w, float power)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, power, true));
    }
};

// 2^(byte - 127) of byte number i of a word; shift = 8 i.
__device__ __forceinline__ float power_of(uint32_t word, uint32_t shift)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_ubfe(word, shift, 8) << 23);
}

// Eight elements as 16-bit floats.
template <class T>
__device__ __forceinline__ w4 widen(w2 x, float power)
{
    return w4{E4M3<T>::low(x[0], power), E4M3<T>::high(x[0], power), E4M3<T>::low(x[1], power), E4M3<T>::high(x[1], power)};
}

// The least e with |x| <= 448 * 2^e for the largest |x| of 32 elements (finite), within the type's limits.
template <class T>
__device__ __forceinline__ int32_t exponent_for(float largest)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, largest);
    const int32_t e = (int32_t)(u >> 23) - 135 + ((u & 0x7FFFFFu) > 0x600000u);   // 448 = 1.75 * 2^8
    return min(max(e, E4M3<T>::kLeast), E4M3<T>::kMost);
}

__device__ __forceinline__ w2 to_e4m3(const float (&y)[8])
{
    w2 out;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], v, true);
        out[w] = (uint32_t)v;
    }
    return out;
}

// Eight finite floats of magnitudes up to 448 * 2^e.
__device__ __forceinline__ w2 narrow_plain(const float (&x)[8], int32_t e)
{
    const float power = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i] * power;
    return to_e4m3(y);
}

// Eight floats as e4m3 elements of exponent e, rounded to nearest even; those that are not finite become NaN.
template <class T>
__device__ __forceinline__ w2 narrow(const float (&x)[8], int32_t e)
{
    const float power = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
    const float limit = e == E4M3<T>::kMost ? 240.0f : 448.0f;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = __builtin_amdgcn_fmed3f(x[i] * power, -limit, limit);
        y[i] = __builtin_isfinite(x[i]) ? s : __builtin_nanf("");
    }
    return to_e4m3(y);
}

}  // namespace kvp

#endif
