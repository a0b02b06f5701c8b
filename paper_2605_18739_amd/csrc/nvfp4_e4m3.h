// 8-bit operands: E4M3 codes with one E8M0 scale (a power of two) for each 128 elements along the contraction axis.
#pragma once

#include "nvfp4_device.h"

namespace nvfp4 {

constexpr int kE4m3Block = 128;

typedef int int8v __attribute__((ext_vector_type(8)));

// The scale byte of a block from the bits of its largest magnitude (finite or not): 127 + e for the smallest e >= -127 with
// amax <= 448 * 2^e.  448 = 1.75 * 2^8, so e is the exponent less 8, and one more where the mantissa is above 1.75: the
// addition carries exactly then.  A block that holds an infinity or NaN gets 255, the scale that is no number.
__device__ __forceinline__ uint32_t e8m0_of_amax(uint32_t amax_bits)
{
    const int byte = (int)((amax_bits + 0x1FFFFFu) >> 23) - 8;
    return amax_bits >= 0x7F800000u ? 255u : (uint32_t)max(byte, 0);
}
// 2^(byte - 127) as the conversions below take it: the byte is the exponent of an fp32 number, and they look at nothing else of it
// (0 is 2^-127, 255 makes every code NaN)
__device__ __forceinline__ float e8m0_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Values that are at most 448 times the scale -> their E4M3 codes, nearest even (NaN: 0x7F with the sign kept).  (Compared with
// scaling by an exact power of two and v_cvt_pk_fp8_f32 on all codes, all midpoints and their neighbours at every scale: the same.)
typedef short short2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ short2v any_pair()          // (both halves get written; a zero would cost a move)
{
    uint32_t w;
#if defined(__HIP_DEVICE_COMPILE__)
    asm("" : "=v"(w));
#else
    w = 0;
#endif
    return __builtin_bit_cast(short2v, w);
}
__device__ __forceinline__ uint32_t e4m3_pack4(float a, float b, float c, float d, float scale)
{
    const short2v w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(any_pair(), a, b, scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true));
}
// two codes in the lower half of a word whose upper half is anything
__device__ __forceinline__ uint32_t e4m3_pack2(float a, float b, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(any_pair(), a, b, scale, false));
}
// two pairs of bf16
__device__ __forceinline__ uint32_t e4m3_pack4(uint32_t ab, uint32_t cd, float scale)
{
    typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
    const short2v w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(any_pair(), __builtin_bit_cast(bf16x2v, ab), scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2v, cd), scale, true));
}

// the larger of m and |v|; NaN if either is (v_maximum3_f32: the older maxima drop it)
__device__ __forceinline__ float abs_max(float m, float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_elementwise_maximum(m, __builtin_fabsf(v));
#else
    return m + v;
#endif
}
// ... as bits that order like unsigned numbers, NaN above all
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32_max(uint32_t v)
{
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true));
}
// maximum over the sixteen lanes of a row of lanes; every lane gets it
__device__ __forceinline__ uint32_t row16_max(uint32_t v)
{
    v = dpp_u32_max<0xB1>(v);
    v = dpp_u32_max<0x4E>(v);
    v = dpp_u32_max<0x141>(v);
    return dpp_u32_max<0x140>(v);
}

__device__ __forceinline__ void unpack8(uint4v v, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16lo_to_f32(v[i]);
        f[2 * i + 1] = bf16hi_to_f32(v[i]);
    }
}
__device__ __forceinline__ uint4v pack8(const float (&f)[8])
{
    return uint4v{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
}
__device__ __forceinline__ uint2v e4m3_pack8(const float (&f)[8], float scale)
{
    return uint2v{e4m3_pack4(f[0], f[1], f[2], f[3], scale), e4m3_pack4(f[4], f[5], f[6], f[7], scale)};
}
__device__ __forceinline__ uint2v e4m3_pack8(uint4v v, float scale) { return uint2v{e4m3_pack4(v.x, v.y, scale), e4m3_pack4(v.z, v.w, scale)}; }
// largest magnitude of eight packed bf16, as the bits of an fp32 number
__device__ __forceinline__ uint32_t absmax8_bits(uint4v v)
{
    return pk_hmax_u16(pk_absmax_u16(pk_absmax_u16(pk_absmax_u16(pk_absmax_u16(0u, v.x), v.y), v.z), v.w)) << 16;
}

// ---- activations of gated layers, in fp32 to about an ulp ---------------------------------------------------------
constexpr int kActSilu = 2, kActGelu = 1;                       // (NVFP4_ACT_*)

// v between two bounds; NaN where v is (v_med3_f32 and the older minima and maxima would give a bound)
__device__ __forceinline__ float clamped(float v, float lo, float hi)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_elementwise_minimum(__builtin_elementwise_maximum(v, lo), hi);
#else
    return v + lo + hi;
#endif
}
// Where the sigmoid is no constant in fp32: it is zero below -87, where it leaves the normal numbers, and one above 104.  (Of a number
// far outside the exponent to base two overflows, and what its rounding drops is infinite.)
__device__ __forceinline__ float sigmoid_within(float x) { return clamped(x, -87.0f, 104.0f); }
// 1 / (1 + exp(-x)), `within` being sigmoid_within(x).  The exponent to base two is taken in two parts: one rounded product would
// cost |x| / 2 ulps.
__device__ __forceinline__ float sigmoid_f32(float x, float within)
{
    constexpr float kLog2e = 1.44269504f, kLog2eLow = 1.92596299e-8f, kLn2 = 0.693147182f;
    const float y = -within, t = y * kLog2e, low = __builtin_fmaf(y, kLog2eLow, __builtin_fmaf(y, kLog2e, -t));
    float e = __builtin_amdgcn_exp2f(t);
    e = __builtin_fmaf(e * low, kLn2, e);
    const float d = 1.0f + e, r = __builtin_amdgcn_rcpf(d), s = __builtin_fmaf(r, __builtin_fmaf(-d, r, 1.0f), r);
    return x < -87.0f ? 0.0f : s;
}
__device__ __forceinline__ float sigmoid_f32(float x) { return sigmoid_f32(x, sigmoid_within(x)); }
// GELU in its tanh form is x sigmoid(z), z = 2 sqrt(2 / pi) (x + 0.044715 x^3).  Beyond 16 the sigmoid is 0 or 1 for good.
constexpr float kGelu1 = 1.59576912f, kGelu3 = 0.0713548163f;   // z = x (kGelu1 + kGelu3 x^2)
__device__ __forceinline__ float gelu_within(float x) { return clamped(x, -16.0f, 16.0f); }
template <int ACT>
__device__ __forceinline__ float activation(float x)
{
    if constexpr (ACT == kActSilu) return x * sigmoid_f32(x);
    else {
        const float c = gelu_within(x);
        return x * sigmoid_f32(c * __builtin_fmaf(kGelu3, c * c, kGelu1));
    }
}
// act(x), and its derivative: sigmoid + x sigmoid (1 - sigmoid) z'.  (At an infinity the derivative is its limit; act(-infinity) is
// NaN, as -infinity times zero is.)
template <int ACT>
__device__ __forceinline__ float activation(float x, float &slope)
{
    if constexpr (ACT == kActSilu) {
        const float c = sigmoid_within(x), s = sigmoid_f32(x, c);
        slope = s * __builtin_fmaf(c, 1.0f - s, 1.0f);
        return x * s;
    } else {
        const float c = gelu_within(x), c2 = c * c, s = sigmoid_f32(c * __builtin_fmaf(kGelu3, c2, kGelu1));
        slope = __builtin_fmaf(c * s, (1.0f - s) * __builtin_fmaf(3.0f * kGelu3, c2, kGelu1), s);
        return x * s;
    }
}

}  // namespace nvfp4
