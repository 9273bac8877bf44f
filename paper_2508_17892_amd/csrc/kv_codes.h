// The two formats of a quantised cache on the device: 32 channels share a scale, a byte b that stands for 2^(b - 127).
#pragma once

#include "ilre_internal.h"

namespace ilre {

typedef __attribute__((ext_vector_type(2))) __bf16 kv_bf16x2;
typedef __attribute__((ext_vector_type(2))) float kv_f32x2;
typedef __attribute__((ext_vector_type(2))) short kv_s16x2;

// Bytes that n channels' codes take, n a multiple of 2.
template <int FMT>
__host__ __device__ constexpr int64_t code_bytes(int64_t n)
{
    return FMT == ILRE_KV_FP8 ? n : n / 2;
}

// The scale's exponent for a block whose largest magnitude is `top`: the smallest e >= -126 with top <= largest code * 2^e (448 = 1.75 * 2^8, 6 = 1.5 * 2^2).  Its byte is e + 127;
// 255 where top is an infinity or a NaN.  Integers only: exponent and fraction of top as they lie in the float.
template <int FMT>
__device__ __forceinline__ unsigned scale_byte(float top)
{
    constexpr unsigned kFraction = FMT == ILRE_KV_FP8 ? 0x600000u : 0x400000u;
    constexpr int kExponent = FMT == ILRE_KV_FP8 ? 8 : 2;
    const unsigned u = __float_as_uint(top), e = u >> 23;  // top >= 0
    const int b = (int)e - kExponent + ((u & 0x7FFFFFu) > kFraction ? 1 : 0);
    return e == 255 ? 255u : (unsigned)(b < 1 ? 1 : b);
}

// (Byte 255 gives an infinity, the exponent that the conversion instructions take for a scale of NaN: whatever the code, zero included, NaN comes out.)
__device__ __forceinline__ float scale_of(unsigned byte) { return __uint_as_float(byte << 23); }

// 2^-(b - 127) for b = 1 .. 254 (the last one as a subnormal number).
__device__ __forceinline__ float inverse_scale(unsigned byte) { return __uint_as_float(byte == 254 ? 0x400000u : (254 - byte) << 23); }

// A float that rounds to 7 bits or fewer as x does: x cut off, its last bit set where anything was left out (rounding to the nearest float first could end up halfway between two
// codes, and then on the other side).
__device__ __forceinline__ float cut_off(double x)
{
    const unsigned long long u = __double_as_longlong(x);
    const unsigned lo = (unsigned)u, rest = lo & 0x1FFFFFFFu;
    const double y = __longlong_as_double((long long)((u & ~0x1FFFFFFFull) | (rest ? 0x20000000ull : 0ull)));
    return (float)y;  // exact, but for subnormal and infinite results
}

// Eight codes of x * inv.
__device__ __forceinline__ uint2 to_fp8(const float (&x)[8], float inv)
{
    unsigned w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        kv_s16x2 r = kv_s16x2{0, 0};
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, x[4 * i] * inv, x[4 * i + 1] * inv, 1.0f, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, x[4 * i + 2] * inv, x[4 * i + 3] * inv, 1.0f, true);
        w[i] = __builtin_bit_cast(unsigned, r);
    }
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ unsigned to_fp4(const float (&x)[8], float inv)
{
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0] * inv, x[1] * inv, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2] * inv, x[3] * inv, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4] * inv, x[5] * inv, 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6] * inv, x[7] * inv, 1.0f, 3);
    return w;
}

// The channels of one word of codes, two at a time, times the scale: fp8 four channels, fp4 eight.  Exact.
template <int FMT, int I>
__device__ __forceinline__ unsigned bf16_pair(unsigned w, float scale)
{
    if constexpr (FMT == ILRE_KV_FP8)
        return __builtin_bit_cast(unsigned, (kv_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, I == 1));
    else
        return __builtin_bit_cast(unsigned, (kv_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, I));
}
template <int FMT, int I>
__device__ __forceinline__ float2 f32_pair(unsigned w, float scale)
{
    kv_f32x2 f;
    if constexpr (FMT == ILRE_KV_FP8)
        f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, I == 1);
    else
        f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, I);
    return make_float2(f[0], f[1]);
}

}  // namespace ilre
