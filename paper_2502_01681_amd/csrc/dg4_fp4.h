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

// The scale of a block from the bits of its largest magnitude (fp32), as a float's bits of which the exponent alone counts: the smallest
// power of two with which that magnitude is at most 7 times it. 7 and not 6, the largest code: up to 7 the nearest code is 6 and no further
// off than a tie between 4 and 6. (Blocks of normal numbers, error in the 2-norm: 11.2 % so, 11.7 % with 6, 11.6 % with anything below 8;
// heavier tails differ by more.) 7 = 1.75 * 2^2: adding 2^21 - 1 to the bits carries into the exponent exactly where the mantissa is above
// 1.75; then two powers are taken off, down to 2^-127. An infinity or a NaN gives something else than FP4_BAD << 23.
__device__ __forceinline__ uint32_t fp4_scale_bits(uint32_t top) { return __builtin_elementwise_sub_sat(top, (2u << 23) - 0x1FFFFFu); }
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t top)
{
    return top >= 0x7F800000u ? FP4_BAD : fp4_scale_bits(top) >> 23;
}
// The conversions take the exponent bits of a scale alone (checked), so 2^-127 is 0. To nearest, ties to even, from 6 on to 6, whatever
// the scale (every bfloat16 number has been compared); a zero keeps its sign.
// (A word before its first codes are put in: any)
__device__ __forceinline__ uint32_t fp4_nothing() { return __builtin_nondeterministic_value(0u); }
template <int SEL> __device__ __forceinline__ uint32_t fp4_put2(uint32_t w, float a, float b, uint32_t scale_bits)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, __uint_as_float(scale_bits), SEL);
}
template <int SEL> __device__ __forceinline__ uint32_t fp4_put2(uint32_t w, uint32_t pair, uint32_t scale_bits)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pair), __uint_as_float(scale_bits), SEL);
}
__device__ __forceinline__ uint32_t fp4_put8(const float* f, uint32_t scale_bits)
{
    uint32_t w = fp4_nothing();
    w = fp4_put2<0>(w, f[0], f[1], scale_bits);
    w = fp4_put2<1>(w, f[2], f[3], scale_bits);
    w = fp4_put2<2>(w, f[4], f[5], scale_bits);
    return fp4_put2<3>(w, f[6], f[7], scale_bits);
}
// The eight codes of a word as numbers, times 2^(byte - 127)
__device__ __forceinline__ void fp4_get8(uint32_t w, uint32_t byte, float* f)
{
    const float scale = __uint_as_float(byte << 23);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
}

// Values of a row that a lane holds as loaded, N = 8 or 16 neighbouring ones (a quarter or half of a block): the largest magnitude as
// bits of fp32, and their codes
template <typename T, int N> struct Values {
    static constexpr int PIECES = N * (int)sizeof(T) / 16;
    uint4 w[PIECES];
    __device__ __forceinline__ void load(const T* p)
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) w[i] = ((const uint4*)p)[i];
    }
    __device__ __forceinline__ void store(T* p) const
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) ((uint4*)p)[i] = w[i];
    }
    __device__ __forceinline__ uint32_t top() const
    {
        u16x2 pairs = { 0, 0 };
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const uint32_t x[4] = { w[i].x, w[i].y, w[i].z, w[i].w };
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (sizeof(T) == 2) pairs = __builtin_elementwise_max(pairs, __builtin_bit_cast(u16x2, x[k] & 0x7FFF7FFFu));
                else t = max(t, x[k] & 0x7FFFFFFFu);
            }
        }
        return sizeof(T) == 2 ? (uint32_t)max(pairs.x, pairs.y) << 16 : t;
    }
    __device__ __forceinline__ void codes(uint32_t scale_bits, uint32_t (&to)[N / 8]) const
    {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            if constexpr (sizeof(T) == 2) {
                uint32_t c = fp4_nothing();
                c = fp4_put2<0>(c, w[i].x, scale_bits);
                c = fp4_put2<1>(c, w[i].y, scale_bits);
                c = fp4_put2<2>(c, w[i].z, scale_bits);
                to[i] = fp4_put2<3>(c, w[i].w, scale_bits);
            } else {
                float f[8];
                Elem<float>::unpack(w[2 * i], w[2 * i + 1], f);
                to[i] = fp4_put8(f, scale_bits);
            }
        }
    }
};
// The largest of two or four neighbouring lanes, which hold a block
template <int LANES> __device__ __forceinline__ uint32_t max_of_lanes(uint32_t t)
{
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xF, 0xF, true));
    if constexpr (LANES == 4) t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xF, 0xF, true));
    return t;
}

// A launch with the status of its own (hipGetLastError takes 0.2 us of a short call's 3, and may return what another call left)
template <typename A> int launch(void (*kernel)(A), dim3 grid, int threads, hipStream_t s, A a)
{
    void* args[] = { &a };
    return (int)hipLaunchKernel((const void*)kernel, grid, dim3((unsigned)threads), args, 0, s);
}

}  // namespace
