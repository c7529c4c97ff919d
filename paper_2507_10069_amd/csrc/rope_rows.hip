// Rotary positions of q and k, and the way of new K and V rows into the 8-bit cache (formulas: include/emm.h,
// include/emm_fp8.h).
//
// Both are bound by the bytes of the rows.  A row is one (token, head); a lane holds 16 of its channels, so that a head of
// 128 is 8 lanes and a wave takes 8 rows at a time.  Of a rotated head they are 8 pairs: channels 8 u .. 8 u + 7 and the 8 that
// are rotary_dim / 2 further up, or 16 in a row where pairs are neighbours.  A token's cosines and sines are made once by
// its wave, a lane for each frequency (at most 64), and reach the lanes that need eight of them through LDS.
#include "fp8_device.h"

namespace emm {

namespace {

using namespace fp8;

constexpr int WAVES = 4;

template <typename T> struct Row8;                       // eight neighbouring channels in memory and in 32 bits
template <> struct Row8<__bf16> {
    static __device__ void load(const __bf16* p, float (&x)[8])
    {
        const bf16x8 v = *(const bf16x8*)p;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
    }
    static __device__ void store(__bf16* p, const float (&x)[8])
    {
        bf16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
        *(bf16x8*)p = v;
    }
    static __device__ float rounded(float x) { return (float)(__bf16)x; }
};
template <> struct Row8<float> {
    static __device__ void load(const float* p, float (&x)[8])
    {
        const float4 a = *(const float4*)p, c = *(const float4*)(p + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = c.x; x[5] = c.y; x[6] = c.z; x[7] = c.w;
    }
    static __device__ void store(float* p, const float (&x)[8])
    {
        *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
        *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
    }
    static __device__ float rounded(float x) { return x; }
};

// cosine and sine of frequency i at a token, times the factor.  The angle is reduced in 64 bits: in turns, less the
// nearest whole number of them.
__device__ inline float2 turn_of(const RopeView& r, int i, long long position)
{
    constexpr double TURNS_PER_RADIAN = 0.15915494309189533577;
    const double turns = (double)position * r.inv_freq[i] * TURNS_PER_RADIAN;
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    return make_float2(c * r.factor, s * r.sine_factor);
}

template <int LANES>                                     // largest of the 4 or 8 lanes that hold a row
__device__ inline uint32_t row_most(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, true));              // quad_perm 1 0 3 2
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, true));              // quad_perm 2 3 0 1
    if constexpr (LANES == 8) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true));   // mirrored in eight
    return x;
}

// rows of a token: K heads, then (QUANT) V heads, then q heads
template <typename T, int D, bool QUANT>
__global__ __launch_bounds__(64 * WAVES) void rope_rows_kernel(BatchView b, RopeView rope, NewRows rows, Fp8Pools pools, int splits)
{
    constexpr int UNITS = D / 16, ROWS = 64 / UNITS;
    __shared__ float2 turns[WAVES][D / 2];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const long long item = (long long)blockIdx.x * WAVES + wave;
    const int t = (int)(item / splits), part = (int)(item - (long long)t * splits);
    if (t >= b.total_new_tokens) return;

    TokenPlace place = {0, -1};
    long long row0 = -1;
    const bool from_batch = rope.rotary_dim > 0 && rope.num_axes == 0;
    if (QUANT || from_batch) {
        place = place_of_token(b, t);
        if (place.slot < 0) return;                      // a row of no request stays as it was
    }
    if (QUANT) row0 = pool_row(b, place);
    if (lane < rope.rotary_dim / 2) {
        long long position = place.slot;
        if (!from_batch) {
            const int axis = (lane >= rope.ends[0] ? 1 : 0) + (lane >= rope.ends[1] ? 1 : 0) + (lane >= rope.ends[2] ? 1 : 0);
            position = rope.positions[(long long)min(axis, rope.num_axes - 1) * b.total_new_tokens + t];
        }
        turns[wave][lane] = turn_of(rope, lane, position);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();

    const int n_k = rows.k != nullptr ? b.num_kv_heads : 0, n_v = QUANT ? b.num_kv_heads : 0, n_q = rows.q != nullptr ? b.num_q_heads : 0;
    const int n_rows = n_k + n_v + n_q, u = lane % UNITS;
    float2 cs[8] = {};
    const bool unit_turns = u < rope.rotary_dim / 16;
    if (unit_turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) cs[i] = turns[wave][8 * u + i];
    }
    for (int base = part * ROWS; base < n_rows; base += splits * ROWS) {
        const int row = base + lane / UNITS;
        const bool valid = row < n_rows, is_k = row < n_k, is_v = !is_k && row < n_k + n_v;
        const int head = is_k ? row : is_v ? row - n_k : row - n_k - n_v;
        const bool turned = unit_turns && !is_v;
        const bool apart = turned && !rope.interleaved;
        const int a0 = apart ? 8 * u : 16 * u, a1 = apart ? rope.rotary_dim / 2 + 8 * u : 16 * u + 8;
        float x[8] = {}, y[8] = {};
        if (valid) {
            const T* src = (is_k ? (const T*)rows.k + t * rows.k_stride : is_v ? (const T*)rows.v + t * rows.v_stride : (const T*)rows.q + t * rows.q_stride) + head * D;
            Row8<T>::load(src + a0, x);
            Row8<T>::load(src + a1, y);
        }
        if (turned) {
            if (rope.interleaved) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = x[2 * i], c = x[2 * i + 1], d = y[2 * i], e = y[2 * i + 1];
                    x[2 * i] = a * cs[i].x - c * cs[i].y;
                    x[2 * i + 1] = c * cs[i].x + a * cs[i].y;
                    y[2 * i] = d * cs[4 + i].x - e * cs[4 + i].y;
                    y[2 * i + 1] = e * cs[4 + i].x + d * cs[4 + i].y;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float a = x[i], c = y[i];
                    x[i] = a * cs[i].x - c * cs[i].y;
                    y[i] = c * cs[i].x + a * cs[i].y;
                }
            }
        }
        if (QUANT && (is_k || is_v)) {
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = Row8<T>::rounded(x[i]);
                y[i] = Row8<T>::rounded(y[i]);
                most = max(most, finite(x[i]) ? __float_as_uint(x[i]) & 0x7fffffffu : 0u);
                most = max(most, finite(y[i]) ? __float_as_uint(y[i]) & 0x7fffffffu : 0u);
            }
            const int byte = scale_byte(row_most<UNITS>(most));
            const float down = down_scale(byte);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = scaled_down(x[i], down);
                y[i] = scaled_down(y[i], down);
            }
            if (valid && row0 >= 0) {
                const long long at = row0 + (long long)head * b.page_size;
                unsigned char* codes = (is_k ? pools.k : pools.v) + at * D;
                *(uint2*)(codes + a0) = make_uint2(pack4(x[0], x[1], x[2], x[3]), pack4(x[4], x[5], x[6], x[7]));
                *(uint2*)(codes + a1) = make_uint2(pack4(y[0], y[1], y[2], y[3]), pack4(y[4], y[5], y[6], y[7]));
                if (u == 0) (is_k ? pools.k_scale : pools.v_scale)[at] = (unsigned char)byte;
            }
        } else if (valid) {
            const int heads = is_k ? b.num_kv_heads : b.num_q_heads;
            T* dst = (T*)(is_k ? rows.k_out : rows.q_out) + ((long long)t * heads + head) * D;
            Row8<T>::store(dst + a0, x);
            Row8<T>::store(dst + a1, y);
        }
    }
}

// 16 codes to the batch's dtype, exact
__device__ inline void widen16(const uint4 c, int byte, __bf16* dst)
{
    const float scale = up_scale(byte);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    bf16x2 v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false);
        v[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
        *(uint4*)(dst + 8 * i) = make_uint4(__builtin_bit_cast(uint32_t, v[4 * i]), __builtin_bit_cast(uint32_t, v[4 * i + 1]),
                                            __builtin_bit_cast(uint32_t, v[4 * i + 2]), __builtin_bit_cast(uint32_t, v[4 * i + 3]));
}
__device__ inline void widen16(const uint4 c, int byte, float* dst)
{
    const float scale = up_scale(byte);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, true);
        *(float4*)(dst + 4 * i) = make_float4(lo[0], lo[1], hi[0], hi[1]);
    }
}

template <typename T, int D>
__global__ __launch_bounds__(64 * WAVES) void kv_gather_fp8_kernel(BatchView b, Fp8Pools pools, T* __restrict__ k_out, T* __restrict__ v_out)
{
    constexpr int UNITS = D / 16, ROWS = 64 / UNITS;
    const int t = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (t >= b.total_new_tokens) return;
    const long long row0 = pool_row(b, place_of_token(b, t));
    if (row0 < 0) return;
    const int u = lane % UNITS;
    for (int row = lane / UNITS; row < 2 * b.num_kv_heads; row += ROWS) {
        const bool is_k = row < b.num_kv_heads;
        const int head = is_k ? row : row - b.num_kv_heads;
        const long long at = row0 + (long long)head * b.page_size;
        const uint4 codes = *(const uint4*)((is_k ? pools.k : pools.v) + at * D + 16 * u);
        const int byte = (is_k ? pools.k_scale : pools.v_scale)[at];
        widen16(codes, byte, (is_k ? k_out : v_out) + ((long long)t * b.num_kv_heads + head) * D + 16 * u);
    }
}

template <typename T, int D>
hipError_t launch_rows(const BatchView& b, const RopeView& rope, const NewRows& rows, const Fp8Pools* pools, hipStream_t stream)
{
    constexpr int splits = 1;
    const long long items = (long long)b.total_new_tokens * splits;
    const dim3 grid((unsigned)((items + WAVES - 1) / WAVES)), block(64 * WAVES);
    if (pools != nullptr) hipLaunchKernelGGL((rope_rows_kernel<T, D, true>), grid, block, 0, stream, b, rope, rows, *pools, splits);
    else hipLaunchKernelGGL((rope_rows_kernel<T, D, false>), grid, block, 0, stream, b, rope, rows, Fp8Pools{}, splits);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_gather(const BatchView& b, const Fp8Pools& pools, void* k_out, void* v_out, hipStream_t stream)
{
    hipLaunchKernelGGL((kv_gather_fp8_kernel<T, D>), dim3((unsigned)(((long long)b.total_new_tokens + WAVES - 1) / WAVES)), dim3(64 * WAVES), 0, stream, b, pools,
                       (T*)k_out, (T*)v_out);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_rows(const BatchView& b, bool bf16, const RopeView& rope, const NewRows& rows, const Fp8Pools* pools, hipStream_t stream)
{
    if (bf16) return b.head_dim == 128 ? launch_rows<__bf16, 128>(b, rope, rows, pools, stream) : launch_rows<__bf16, 64>(b, rope, rows, pools, stream);
    return b.head_dim == 128 ? launch_rows<float, 128>(b, rope, rows, pools, stream) : launch_rows<float, 64>(b, rope, rows, pools, stream);
}

hipError_t launch_kv_gather_fp8(const BatchView& b, bool bf16, const Fp8Pools& pools, void* k_out, void* v_out, hipStream_t stream)
{
    if (bf16) return b.head_dim == 128 ? launch_gather<__bf16, 128>(b, pools, k_out, v_out, stream) : launch_gather<__bf16, 64>(b, pools, k_out, v_out, stream);
    return b.head_dim == 128 ? launch_gather<float, 128>(b, pools, k_out, v_out, stream) : launch_gather<float, 64>(b, pools, k_out, v_out, stream);
}

}  // namespace emm
