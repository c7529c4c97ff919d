// The 8-bit cache's format on the device (see include/emm_fp8.h), and where a packed token's slot is.
#pragma once

#include "fp8_internal.h"

namespace emm {
namespace fp8 {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int LEAST_EXPONENT = -117;         // every value of such a row is still a normal bf16,
constexpr int MOST_EXPONENT = 119;           // and of such a row a finite one: 448 * 2^119 = 2.98e38
constexpr int BIAS = 127;                    // of the scale byte

// A row's scale byte from the bits of its largest finite |x|: e + 127 with e the least integer -117 .. 119 such that
// most <= 448 * 2^e, or 119; 448 = 1.75 * 2^8.
__device__ inline int scale_byte(uint32_t most_bits)
{
    const int e = (int)(most_bits >> 23) - BIAS - 8 + ((most_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return min(max(e, LEAST_EXPONENT), MOST_EXPONENT) + BIAS;
}
// 2^(127 - byte): the factor before rounding; exact (bytes are 10 .. 246)
__device__ inline float down_scale(int byte) { return __uint_as_float((uint32_t)(2 * BIAS - byte) << 23); }
// 2^(byte - 127)
__device__ inline float up_scale(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// a row's value in its scale: at most 448 in magnitude, or NaN
__device__ inline float scaled_down(float x, float down)
{
    const bool is_finite = (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u;
    return is_finite ? fminf(fmaxf(x * down, -448.0f), 448.0f) : __builtin_nanf("");
}

__device__ inline bool finite(float x) { return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u; }

// four scaled values to four codes (nearest even; at most 448 in magnitude, or NaN)
__device__ inline uint32_t pack4(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// A packed token's request and slot.  Wave-uniform.  The last request whose first token is not behind t, among 64 that the
// lanes look at together; `slot` < 0: the token belongs to no request.
struct TokenPlace {
    int req;
    long long slot;
};
__device__ inline TokenPlace place_of_token(const BatchView& b, int t)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = b.num_reqs;
    while (hi - lo > 64) {
        const int mid = (lo + hi) >> 1;
        if (b.cu_new_lens[mid] <= t) lo = mid; else hi = mid;
    }
    const int mine = min(lo + lane, hi - 1);
    const int cu = b.cu_new_lens[mine], prefix = b.prefix_lens[mine], count = b.new_lens[mine];
    const unsigned long long not_after = __builtin_amdgcn_ballot_w64(lo + lane < hi && cu <= t);
    const int at = not_after == 0 ? 0 : 63 - __builtin_clzll(not_after);
    const int j = t - __builtin_amdgcn_readlane(cu, at);
    const bool in_request = not_after != 0 && j < __builtin_amdgcn_readlane(count, at);
    TokenPlace p;
    p.req = lo + at;
    p.slot = in_request ? (long long)__builtin_amdgcn_readlane(prefix, at) + j : -1;
    return p;
}
// The pool row (of KV head 0; heads are page_size rows apart) that holds a slot, or -1 where the table has none: nothing is
// written or read there.
__device__ inline long long pool_row(const BatchView& b, const TokenPlace& p)
{
    if (p.slot < 0 || p.slot >= (long long)b.max_pages * b.page_size) return -1;
    const int slot = (int)p.slot;
    const int page = b.page_table[(long long)p.req * b.max_pages + (slot >> (4 + b.page_shift))];
    if (page < 0 || page >= b.num_pages) return -1;
    return (long long)page * b.num_kv_heads * b.page_size + (slot & (b.page_size - 1));
}

}  // namespace fp8
}  // namespace emm
