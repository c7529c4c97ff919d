// What the two attention kernels over the 8-bit cache share: sums over lanes, the format's NaN.
//
// Both make K's codes bf16, in their row's scale (v_cvt_scalef32_pk_bf16_fp8, exact), for products in bf16.  The matrix instructions
// that take the codes as they are would save that, but keep a sum of 8-bit products only to about 2^-16 of the largest of them (128
// random products of up to 5e4: off by 1.8, in bf16 by 0.001), which makes the scores 25 times less exact than 32 bits are.
#pragma once

#include "attn_bf16_common.h"
#include "fp8_device.h"

namespace emm {
namespace fp8 {

using bf16attn::pair_max;
using bf16attn::pair_sum;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int HEAD_DIM = 128;
constexpr float LN2 = 0.69314718055994530942f, LOG2E = 1.44269504088896340736f;

// x with the lane 16 further (within 32), in both lanes; with the lane 32 further: pair_max, pair_sum
__device__ inline float max16(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum16(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
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
