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

// ---- activations of gated layers ------------------------------------------------------------------------------------
// In fp32, u = 2^-24 (these steps with correctly rounded exponentials and reciprocals, over 10^6 gates): act within 4 u of itself, down
// to where its sigmoid leaves the normal numbers (about e^-87) and is taken as zero; the derivative within 4 u (GELU) and 16 u (SiLU: around
// 16, where 1 - s is the difference of nearly equal numbers).
constexpr int kActSilu = 2, kActGelu = 1;                       // (NVFP4_ACT_*)

// v between two bounds; a bound where v is NaN
__device__ __forceinline__ float bounded(float v, float lo, float hi) { return __builtin_amdgcn_fmed3f(v, lo, hi); }
// ... and NaN there, at one instruction more
__device__ __forceinline__ float clamped(float v, float lo, float hi)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_elementwise_minimum(__builtin_elementwise_maximum(v, lo), hi);
#else
    return v + lo + hi;
#endif
}
// 1 / (1 + exp(-x)), `within` being x between these: the sigmoid is zero below, where it leaves the normal numbers, and one above.  (Of a
// number far outside the exponent to base two overflows, and what its rounding drops is infinite.)  The exponent comes in two parts:
// one rounded product x log2(e) would cost |x| / 2 ulps.
constexpr float kSigmoidLow = -87.0f, kSigmoidHigh = 104.0f, kLn2 = 0.693147182f;
__device__ __forceinline__ float sigmoid_f32(float x, float within)
{
    constexpr float kLog2e = 1.44269504f, kLog2eLow = 1.92596299e-8f;
    const float y = -within, t = y * kLog2e, low = __builtin_fmaf(y, kLog2eLow, __builtin_fmaf(y, kLog2e, -t));
    float e = __builtin_amdgcn_exp2f(t);
    e = __builtin_fmaf(e * low, kLn2, e);
    const float d = 1.0f + e, r = __builtin_amdgcn_rcpf(d), s = __builtin_fmaf(r, __builtin_fmaf(-d, r, 1.0f), r);
    return x < kSigmoidLow ? 0.0f : s;
}
// GELU in its tanh form is x sigmoid(z), z = 2 sqrt(2 / pi) (x + 0.044715 x^3) = x (kGelu1 + kGelu3 x^2).  Beyond kGeluEnd the sigmoid is
// 0 or 1 for good.  For negative z it is about e^z, which turns z's relative error into |z| times as much (an fp32 z: 80 u at -7, 200 u
// at -10).  So the exponent to base two, -z log2(e) = -c p, p = K1 + K3 c^2, carries what each step drops: c^2's remainder, p's (the upper
// part of K1 has twelve bits: p - K1 is exact, whichever of the two terms is larger) and the product's.
constexpr float kGelu1 = 1.59576912f, kGelu3 = 0.0713548163f, kGeluEnd = 16.0f;
// sigmoid(z) at c (within kGeluEnd), c2 = c^2; e = e^-z, which may be infinite: the reciprocal is zero then (a step after it would be NaN)
__device__ __forceinline__ float gelu_sigmoid(float c, float c2, float &e)
{
    constexpr float kUp1 = 2.30224609375f, kLow1 = -3.7895606510574e-05f, kUp3 = 0.10294324159622192f, kLow3 = -2.016198319410023e-09f;     // 2 sqrt(2 / pi) log2(e), and 0.044715 of it
    const float p = __builtin_fmaf(kUp3, c2, kUp1), p_low = __builtin_fmaf(kUp3, c2, kUp1 - p) + __builtin_fmaf(kLow3, c2, kLow1);
    const float rest = __builtin_fmaf(kUp3, __builtin_fmaf(c, c, -c2), p_low), t = -c * p, minus_low = __builtin_fmaf(c, rest, __builtin_fmaf(c, p, t));
    e = __builtin_amdgcn_exp2f(t) * __builtin_fmaf(minus_low, -kLn2, 1.0f);
    return __builtin_amdgcn_rcpf(1.0f + e);
}
// act(x).  (A NaN that the bounds take away comes back with the factor x.)
template <int ACT>
__device__ __forceinline__ float activation(float x)
{
    if constexpr (ACT == kActSilu) return x * sigmoid_f32(x, bounded(x, kSigmoidLow, kSigmoidHigh));
    else {
        float e;
        const float c = bounded(x, -kGeluEnd, kGeluEnd);
        return x * gelu_sigmoid(c, c * c, e);
    }
}
// act(x), and its derivative: sigmoid + x sigmoid (1 - sigmoid) z'.  (At an infinity the derivative is its limit; act(-infinity) is
// NaN, as -infinity times zero is.)
template <int ACT>
__device__ __forceinline__ float activation(float x, float &slope)
{
    if constexpr (ACT == kActSilu) {
        const float c = clamped(x, kSigmoidLow, kSigmoidHigh), s = sigmoid_f32(x, c);
        slope = s * __builtin_fmaf(c, 1.0f - s, 1.0f);
        return x * s;
    } else {
        float e;
        const float c = clamped(x, -kGeluEnd, kGeluEnd), c2 = c * c, s = gelu_sigmoid(c, c2, e);
        slope = __builtin_fmaf(c * s, fminf(e, 1e38f) * s * __builtin_fmaf(3.0f * kGelu3, c2, kGelu1), s);      // (1 - s = e s; s is zero where e is infinite)
        return x * s;
    }
}

}  // namespace nvfp4
