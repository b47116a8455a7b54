// Blocks of 32 numbers in 4 bits under one power of two, for the kernels that write, read and multiply them: codes 0 .. 15 (a
// sign bit over the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6), two to a byte, the first in the low half; the power of two as
// exponent + 127, 255 for a block with an infinity or a NaN. The element and scale formats are those that gfx950's matrix cores
// and conversions take.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dg4_device.h"

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t FP4_BAD = 255;                 // scale byte of a block that is not finite

// The scale byte of a block from the bits of its largest magnitude (fp32): the smallest power of two with which that is at most 7
// times it. 7 and not 6, the largest code: up to 7 the nearest code is 6 and no further off than a tie between 4 and 6. (Blocks
// of normal numbers, error in the 2-norm: 11.2 % so, 11.7 % with 6, 11.6 % with anything below 8; heavier tails differ by more.)
// 7 = 1.75 * 2^2: adding what the mantissa may miss to the next power carries into the exponent exactly where it is above 1.75.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t top)
{
    const int e = (int)((top + 0x1FFFFFu) >> 23) - 2;
    return top >= 0x7F800000u ? FP4_BAD : (uint32_t)(e > 0 ? e : 0);
}
// 2^(byte - 127) (0: a subnormal number; 255: NaN)
__device__ __forceinline__ float fp4_scale_value(uint32_t byte)
{
    const uint32_t bits = byte == 0 ? 0x00400000u : byte << 23;
    return __uint_as_float(byte == FP4_BAD ? 0x7FC00000u : bits);
}

// The conversions take a scale's exponent bits alone: byte << 23 is right for 0 too. To nearest, ties to even, from 6 on to 6,
// whatever the scale (every bfloat16 number has been compared); a zero keeps its sign.
template <int SEL> __device__ __forceinline__ uint32_t fp4_put2(uint32_t w, float a, float b, uint32_t byte)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, __uint_as_float(byte << 23), SEL);
}
template <int SEL> __device__ __forceinline__ uint32_t fp4_put2(uint32_t w, uint32_t pair, uint32_t byte)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pair), __uint_as_float(byte << 23), SEL);
}
__device__ __forceinline__ uint32_t fp4_put8(const float* f, uint32_t byte)
{
    uint32_t w = 0;
    w = fp4_put2<0>(w, f[0], f[1], byte);
    w = fp4_put2<1>(w, f[2], f[3], byte);
    w = fp4_put2<2>(w, f[4], f[5], byte);
    return fp4_put2<3>(w, f[6], f[7], byte);
}
// The eight codes of a word as numbers, times 2^(byte - 127)
__device__ __forceinline__ void fp4_get8(uint32_t w, uint32_t byte, float* f)
{
    const float scale = __uint_as_float(byte << 23);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
}

// Eight neighbouring values of a row, a quarter of a block, as loaded; the largest magnitude as bits of fp32; their codes
template <typename T> struct Eighth;
template <> struct Eighth<float> {
    uint4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = ((const uint4*)p)[0]; b = ((const uint4*)p)[1]; }
    __device__ __forceinline__ uint32_t top() const
    {
        const uint32_t w[8] = { a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w };
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, w[i] & 0x7FFFFFFFu);
        return t;
    }
    __device__ __forceinline__ uint32_t codes(uint32_t byte) const
    {
        float f[8];
        Elem<float>::unpack(a, b, f);
        return fp4_put8(f, byte);
    }
};
template <> struct Eighth<bf16_t> {
    uint4 a;
    __device__ __forceinline__ void load(const bf16_t* p) { a = *(const uint4*)p; }
    __device__ __forceinline__ uint32_t top() const
    {
        const uint32_t w[4] = { a.x, a.y, a.z, a.w };
        u16x2 t = { 0, 0 };
#pragma unroll
        for (int i = 0; i < 4; ++i) t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
        return (uint32_t)max(t.x, t.y) << 16;
    }
    __device__ __forceinline__ uint32_t codes(uint32_t byte) const
    {
        uint32_t w = 0;
        w = fp4_put2<0>(w, a.x, byte);
        w = fp4_put2<1>(w, a.y, byte);
        w = fp4_put2<2>(w, a.z, byte);
        return fp4_put2<3>(w, a.w, byte);
    }
};
// The largest of four neighbouring lanes, which hold a block
__device__ __forceinline__ uint32_t max_of_4_lanes(uint32_t t)
{
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xF, 0xF, true));
    return max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xF, 0xF, true));
}

}  // namespace
