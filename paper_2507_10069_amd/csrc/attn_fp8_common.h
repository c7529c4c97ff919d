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

__device__ inline float saturated(float x) { return x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f); }

// Four values of a row of q, in its scale, as two parts: the nearest codes, and 16 times what they leave.  A bf16 has
// eight significant bits and a code four, so the two hold it whole, down to 2^-22 of the row's largest value.
struct QCodes { uint32_t high, low; };
__device__ inline QCodes split4(const float (&x)[4], float down)
{
    float a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = finite(x[i]) ? x[i] * down : __builtin_nanf("");
    QCodes c;
    c.high = pack4(saturated(a[0]), saturated(a[1]), saturated(a[2]), saturated(a[3]));
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c.high, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c.high, true);
    c.low = pack4(saturated((a[0] - lo[0]) * 16.0f), saturated((a[1] - lo[1]) * 16.0f), saturated((a[2] - hi[0]) * 16.0f), saturated((a[3] - hi[1]) * 16.0f));
    return c;
}
constexpr int LOW_PART_SCALE = -4;                       // of the scale byte: the low part's 1 / 16

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
