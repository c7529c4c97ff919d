// What the two attention kernels over the 8-bit cache share: q's operands, the plan's scan, the format's NaN.
#pragma once

#include "fp8_device.h"

namespace emm {
namespace fp8 {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int HEAD_DIM = 128;
constexpr float LN2 = 0.69314718055994530942f, LOG2E = 1.44269504088896340736f;

// The scale byte of a row of q from the bits of its largest |x|; NaN's where a value is not finite, and then every score of the
// row is NaN.
__device__ inline int q_scale_byte(uint32_t most_bits) { return most_bits < 0x7f800000u ? scale_byte(most_bits) : 0xff; }
// The largest |x| of the pairs of a row, as bits of 32
template <int N>
__device__ inline uint32_t most_of(const uint32_t (&pairs)[N])
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 most = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, pairs[i] & 0x7fff7fffu));
    return (uint32_t)max(most[0], most[1]) << 16;
}
// Four values of a row of q as two parts: the nearest codes in the row's scale, and those of 16 times what they leave.  A
// bf16 has eight significant bits and a code four, so the two hold it whole from 2^-6 in the row's scale on, where the low part's
// steps are 2^-13: from 2^-13 of the row's largest value, which is above 224 there.  Smaller ones are off by half a step, 2^-21 of it.
constexpr int LOW_PART_SCALE = -4;                       // of the scale byte: the low part's 1 / 16
struct QCodes { uint32_t high, low; };
__device__ inline QCodes split4(uint32_t pair0, uint32_t pair1, int byte)
{
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    const float scale = up_scale(byte), low_scale = up_scale(byte + LOW_PART_SCALE);
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, pair0), scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, pair1), scale, true);
    QCodes c;
    c.high = __builtin_bit_cast(uint32_t, w);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.high, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.high, scale, true);
    s16x2 v = {0, 0};
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, __uint_as_float(pair0 << 16) - a[0], __uint_as_float(pair0 & 0xffff0000u) - a[1], low_scale, false);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, __uint_as_float(pair1 << 16) - d[0], __uint_as_float(pair1 & 0xffff0000u) - d[1], low_scale, true);
    c.low = __builtin_bit_cast(uint32_t, v);
    return c;
}

// x with the lane 16 further (within 32), and with the lane 32 further, in both lanes
__device__ inline float max16(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float max32(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum16(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline float sum32(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// a byte's top bit where a word's byte is a NaN code
__device__ inline uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// running sums over the wave's lanes, inclusive
__device__ inline int scan64(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);      // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);     // row 0's sum to row 1, row 2's to row 3,
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);     // and row 1's to rows 2 and 3
    return x;
}

}  // namespace fp8
}  // namespace emm
