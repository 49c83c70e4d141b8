// Rows of the 8-bit cache: a row's scale and codes, and what they stand for.
//
//   element = code * 2^e,  e the least number >= -100 with max |x| <= M 2^e (M = 448 or 127), at most 100
//
// The power of two makes x / 2^e and code * 2^e exact, so that the code's own rounding is the only one: what a row stands for is a bf16 number, the
// operand of the attention's products, and reading a row back and quantising it again gives the same row.  A scale of 32
// bits with max |x| on the largest code would leave integer codes half a bit more on average, nothing to 8-bit floats.
#pragma once

#include "attn.cuh"

#include <cuda_fp16.h>

namespace wkv {

constexpr int kLeastExponent = -100, kMostExponent = 100;
constexpr int kScaleBias = 127, kScaleNan = 255;

// |x| as bits: of these the largest is the row's largest, infinity beyond all numbers and NaN beyond that
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// the scale byte of a row whose largest magnitude has these bits
__device__ __forceinline__ int scale_byte(unsigned most, int kind)
{
    if (most >= 0x7f800000u) return kScaleNan;
    // M = 1.75 * 2^8 or 1.984375 * 2^6: a mantissa above M's takes the next power
    const unsigned frac = kind == kE4m3 ? 0x600000u : 0x7e0000u;
    const int top = kind == kE4m3 ? 8 : 6, e = (int)((most + (0x7fffffu - frac)) >> 23) - 127 - top;
    return min(max(e, kLeastExponent), kMostExponent) + kScaleBias;
}
// 2^e and 2^-e of a scale byte that a call has written (27 .. 227); 0 for a NaN row's codes
__device__ __forceinline__ float scale_inverse(int byte) { return byte == kScaleNan ? 0.f : __uint_as_float((unsigned)(254 - byte) << 23); }
// 2^(byte - 127) of any byte, NaN of 255
__device__ __forceinline__ float scale_value(int byte)
{
    return byte == kScaleNan ? __uint_as_float(0x7fffffffu) : (byte == 0 ? __uint_as_float(0x400000u) : __uint_as_float((unsigned)byte << 23));
}

// the larger of two magnitudes, NaN where one is (the instruction takes |x| as it stands)
__device__ __forceinline__ float largest_nan(float top, float x)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(top), "f"(fabsf(x)));
    return r;
}

// Codes of N elements, N a power of two, four to a word; byte: the row's scale.  Integers: in 1.5 * 2^23 + x / 2^e, rounded once, the low byte is the
// code.  Only rows at the largest exponent can pass the largest code, and a NaN row's codes are zeros: those come first.
__device__ __forceinline__ unsigned two_floats(float lo, float hi)
{
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int N>
__device__ __forceinline__ void quantise(const float *from, unsigned *to, int byte, int kind)
{
    const float inverse = scale_inverse(byte);
    float v[N < 4 ? 4 : N];
#pragma unroll
    for (int i = 0; i < (N < 4 ? 4 : N); ++i) v[i] = i < N ? from[i] : 0.f;
    if (byte >= kScaleBias + kMostExponent) {
        const float most = byte == kScaleNan ? 0.f : (kind == kE4m3 ? 448.f : 127.f) * scale_value(byte);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = byte == kScaleNan ? 0.f : fminf(fmaxf(v[i], -most), most);
    }
    if (kind == kE4m3) {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            to[i / 4] = two_floats(v[i] * inverse, v[i + 1] * inverse) | two_floats(v[i + 2] * inverse, v[i + 3] * inverse) << 16;
    } else {
        auto whole = [&](float x) { return __float_as_uint(fmaf(x, inverse, 12582912.f)); };
#pragma unroll
        for (int i = 0; i < N; i += 4)
            to[i / 4] = __byte_perm(__byte_perm(whole(v[i]), whole(v[i + 1]), 0x0040), __byte_perm(whole(v[i + 2]), whole(v[i + 3]), 0x0040), 0x5410);
    }
}

// Codes of four elements as two pairs of f16, exactly.  Integers: with the sign bit flipped they count from 0 to 255, as the low byte of an f16
// in 1024 .. 1279, from which 1152 is taken.
template <int KIND>
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    if (KIND == kE4m3) {
        asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\tcvt.rn.f16x2.e4m3x2 %1, y;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
    } else {
        w ^= 0x80808080u;
        lo = __byte_perm(w, 0x64646464u, 0x4140);
        hi = __byte_perm(w, 0x64646464u, 0x4342);
        const uint32_t by = 0x64806480u;
        asm("sub.f16x2 %0, %0, %1;" : "+r"(lo) : "r"(by));
        asm("sub.f16x2 %0, %0, %1;" : "+r"(hi) : "r"(by));
    }
}
// four codes as they stand, without their scale
template <int KIND>
__device__ __forceinline__ float4 codes_to_float(unsigned w)
{
    uint32_t lo, hi;
    codes_to_f16<KIND>(w, lo, hi);
    const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&lo)), y = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
    return make_float4(x.x, x.y, y.x, y.y);
}
__device__ __forceinline__ float4 codes_to_float(unsigned w, int kind) { return kind == kE4m3 ? codes_to_float<kE4m3>(w) : codes_to_float<kI8>(w); }
// Two pairs of bf16: four codes times 2^e, exactly.  Where 2^e is an f16 (kLeastF16 .. kMostF16), by a multiply-add of f16 into fp32 per element: integers
// keep the 1152 that they are too large by (codes_to_f16) until then.
constexpr int kLeastF16 = kScaleBias - 24, kMostF16 = kScaleBias + 15;
__device__ __forceinline__ uint32_t pack_pair_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int KIND>
__device__ __forceinline__ uint2 codes_to_bf16(unsigned w, float by)
{
    const float4 x = codes_to_float<KIND>(w);
    return make_uint2(pack_pair_bf16(x.x * by, x.y * by), pack_pair_bf16(x.z * by, x.w * by));
}
template <int KIND>
struct F16Scale {
    unsigned short by;
    float more;
    __device__ __forceinline__ explicit F16Scale(float s)
    {
        asm("cvt.rn.f16.f32 %0, %1;" : "=h"(by) : "f"(s));
        more = KIND == kI8 ? -1152.f * s : 0.f;
    }
    __device__ __forceinline__ uint32_t pair(uint32_t x) const
    {
        float lo, hi;
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tfma.rn.f32.f16 %0, a, %3, %4;\n\tfma.rn.f32.f16 %1, b, %3, %4;\n\t}"
            : "=f"(lo), "=f"(hi) : "r"(x), "h"(by), "f"(more));
        return pack_pair_bf16(lo, hi);
    }
    __device__ __forceinline__ uint2 four(uint32_t w) const
    {
        if (KIND == kI8) {
            w ^= 0x80808080u;
            return make_uint2(pair(__byte_perm(w, 0x64646464u, 0x4140)), pair(__byte_perm(w, 0x64646464u, 0x4342)));
        }
        uint32_t lo, hi;
        codes_to_f16<KIND>(w, lo, hi);
        return make_uint2(pair(lo), pair(hi));
    }
};

}  // namespace wkv
