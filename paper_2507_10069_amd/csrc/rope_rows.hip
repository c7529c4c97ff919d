// Rotary positions of q and k, norms of their heads before that, and the way of new K and V rows into a cache (formulas:
// include/emm.h, include/emm_fp8.h, include/emm_step.h).
//
// All are bound by the bytes of the rows.  A row is one (token, head); a lane holds 16 of its channels, so that a head of
// 128 is 8 lanes and a wave takes 8 rows at a time.  Of a rotated head they are 8 pairs: channels 8 u .. 8 u + 7 and the 8 that
// are rotary_dim / 2 further up, or 16 in a row where pairs are neighbours.  A token's cosines and sines are made once by
// its wave, a lane for each frequency (at most 64), and reach the lanes that need eight of them through LDS.
//
// Norms add a sum of squares over the lanes of a row, which travel by DPP, and 16 weights a lane, which stay in registers while a wave is at q's rows.
//
// Measured, of bytes read and written: 4096 tokens of 28 + 4 heads of 128 in bf16 rotated in 12.4 us (67 MB, 5.4 TB/s: they fit the
// last-level cache), with norms 13.1; 42500 tokens of 32 + 8 heads with norms, rotation and the write 207 us (1.07 GB, 5.2 TB/s, what a large copy reaches),
// into the 8-bit cache 190 (0.98 GB, 5.2 TB/s), with heads of 64 108 (0.54 GB, 4.9 TB/s), 4096 such tokens normed and rotated 9.9;
// 46000 tokens' K and V of 8 heads quantised in 57 us (284 MB, 5.0 TB/s), 35000 slots
// of 4 heads read back in 24.2 us (108 MB, 4.5 TB/s).  64 tokens' rotation and write takes 3.9 us on the card, with norms into bf16 3.5, into 8 bits 3.9, an empty kernel 1.7;
// what a decode step waits for is the launch.
#include "fp8_device.h"
#include "step_internal.h"

#include <type_traits>

namespace emm {

namespace {

using namespace fp8;

constexpr int WAVES = 4;
constexpr long long STREAM_BYTES = 96ll << 20;           // codes and values: a call that does not fit the last-level cache next to others
constexpr int MOST_SPLIT = 4096;                         // waves: half of what the chip holds at once (64 tokens 3.9 us, and 5.7 with a wave each, 512
                                                         // 5.0 and 6.3; 2048, which would be 10240 waves, 9.9 so and 11.4 split)

template <typename T> struct Row8;                       // eight neighbouring channels: as they lie in memory, and in 32 bits
template <> struct Row8<__bf16> {
    typedef bf16x8 Raw;
    static __device__ Raw load(const __bf16* p) { return *(const bf16x8*)p; }
    static __device__ void widen(const Raw& v, float (&x)[8])
    {
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
    struct Raw { float4 a, b; };
    static __device__ Raw load(const float* p) { return {*(const float4*)p, *(const float4*)(p + 4)}; }
    static __device__ void widen(const Raw& v, float (&x)[8])
    {
        x[0] = v.a.x; x[1] = v.a.y; x[2] = v.a.z; x[3] = v.a.w;
        x[4] = v.b.x; x[5] = v.b.y; x[6] = v.b.z; x[7] = v.b.w;
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

// A pair's two values.  What is fused is written out, so that the kernels with and without the cache round alike.
__device__ inline float turned_a(float a, float b, float2 cs) { return fmaf(a, cs.x, -(b * cs.y)); }
__device__ inline float turned_b(float a, float b, float2 cs) { return fmaf(b, cs.x, a * cs.y); }

template <int LANES>                                     // largest of the 4 or 8 lanes that hold a row
__device__ inline uint32_t row_most(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, true));              // quad_perm 1 0 3 2
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, true));              // quad_perm 2 3 0 1
    if constexpr (LANES == 8) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true));   // mirrored in eight
    return x;
}

template <int LANES>                                     // sum over them
__device__ inline float row_sum(float x)
{
    auto of = [](float v, auto ctrl) { return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
    x += of(x, std::integral_constant<int, 0xb1>{});
    x += of(x, std::integral_constant<int, 0x4e>{});
    if constexpr (LANES == 8) x += of(x, std::integral_constant<int, 0x141>{});
    return x;
}

// 1 / sqrt(mean(x^2) + eps) of a row, of which this lane holds 16 channels.  Squares of |x| from 1.8e19 on pass the range of 32 bits, or their mean
// with an eps near its end: such a row is taken again in units of 2^70, so that the squares of all finite values add up to less than 2^124.
template <int LANES>
__device__ inline float row_norm(const float (&x)[8], const float (&y)[8], float eps)
{
    constexpr float MEAN = 1.0f / (16 * LANES);
    auto squares = [&](float unit) {
        float a = 0.f, c = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            a = fmaf(x[i] * unit, x[i] * unit, a);
            c = fmaf(y[i] * unit, y[i] * unit, c);
        }
        return row_sum<LANES>(a + c);
    };
    const float mean = fmaf(squares(1.0f), MEAN, eps);
    float norm = __builtin_amdgcn_rsqf(mean);
    if (!(mean < __builtin_inff())) {
        constexpr float UNIT = 0x1p-70f;
        norm = __builtin_amdgcn_rsqf(fmaf(squares(UNIT), MEAN, eps * UNIT * UNIT)) * UNIT;
    }
    return norm;
}

// waves that share a token's rows
struct Splits {
    int n;
    Divisor by;
};
enum Cache { NO_CACHE, FP8, PLAIN /* in the batch's dtype */ };

// rows of a token: K heads, then (with a cache) V heads, then q heads
template <typename T, int D, int CACHE, bool ROPE, bool NORM>
__device__ __forceinline__ void do_rows(BatchView b, RopeView rope, NewRows rows, Fp8Pools pools, PlainPools plain, NormView norm, Splits split)
{
    constexpr bool QUANT = CACHE == FP8, CACHED = CACHE != NO_CACHE;
    constexpr int UNITS = D / 16, ROWS = 64 / UNITS;
    __shared__ float2 turns[WAVES][D / 2];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int item = blockIdx.x * WAVES + wave, splits = split.n;        // (at most 2^25 and a workgroup's)
    const int t = split.by.quotient(item), part = item - t * splits;
    if (t >= b.total_new_tokens) return;

    const int n_k = rows.k != nullptr ? b.num_kv_heads : 0, n_v = CACHED ? b.num_kv_heads : 0, n_q = rows.q != nullptr ? b.num_q_heads : 0;
    const int n_rows = n_k + n_v + n_q, u = lane % UNITS;
    const bool unit_turns = ROPE && u < rope.rotary_dim / 16;
    // a pass: 16 channels of one of the ROWS rows from `base` on, in two eights at a0 and a1
    struct Place {
        int head, a0, a1;
        bool valid, is_k, is_v, turned;
    };
    auto place_in = [&](int base) -> Place {
        Place p;
        const int row = base + lane / UNITS;
        p.valid = row < n_rows;
        p.is_k = row < n_k;
        p.is_v = !p.is_k && row < n_k + n_v;
        p.head = p.is_k ? row : p.is_v ? row - n_k : row - n_k - n_v;
        p.turned = unit_turns && !p.is_v;
        const bool apart = p.turned && !rope.interleaved;
        p.a0 = apart ? 8 * u : 16 * u;
        p.a1 = apart ? rope.rotary_dim / 2 + 8 * u : 16 * u + 8;
        return p;
    };
    typename Row8<T>::Raw raw0 = {}, raw1 = {};
    auto ask = [&](const Place& p) {
        if (p.valid) {
            const T* src = (p.is_k ? (const T*)rows.k + t * rows.k_stride : p.is_v ? (const T*)rows.v + t * rows.v_stride : (const T*)rows.q + t * rows.q_stride) + p.head * D;
            raw0 = Row8<T>::load(src + p.a0);
            raw1 = Row8<T>::load(src + p.a1);
        }
    };
    ask(place_in(part * ROWS));                          // travels while it is worked out where it goes and how far it turns

    TokenPlace place = {0, -1};
    long long row0 = -1;
    const bool from_batch = ROPE && rope.num_axes == 0, given = CACHED && norm.slots != nullptr;
    if ((CACHED && !given) || from_batch) {
        place = place_of_token(b, t);
        if (place.slot < 0 && ((!ROPE && !NORM) || from_batch)) return;  // a row of no request stays as it was; with a given position its q is turned
    }
    if (given) {
        const long long slot = norm.slots[t], page = slot >> (4 + b.page_shift);
        if (slot >= 0 && page < b.num_pages) row0 = page * b.num_kv_heads * b.page_size + (slot & (b.page_size - 1));
    } else if (CACHED) {
        row0 = pool_row(b, place);
    }
    if (ROPE && lane < rope.rotary_dim / 2) {
        long long position = place.slot;
        if (!from_batch) {
            const int axis = (lane >= rope.ends[0] ? 1 : 0) + (lane >= rope.ends[1] ? 1 : 0) + (lane >= rope.ends[2] ? 1 : 0);
            position = rope.positions[(long long)min(axis, rope.num_axes - 1) * b.total_new_tokens + t];
        }
        turns[wave][lane] = turn_of(rope, lane, position);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();

    float2 cs[8] = {};
    if (unit_turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) cs[i] = turns[wave][8 * u + i];
    }
    float wx[8] = {}, wy[8] = {};                            // weights of the lane's channels
    for (int base = part * ROWS; base < n_rows; base += splits * ROWS) {
        const Place p = place_in(base);
        const bool valid = p.valid, is_k = p.is_k, is_v = p.is_v, turned = p.turned;
        const int head = p.head, a0 = p.a0, a1 = p.a1;
        if (base != part * ROWS) ask(p);
        float x[8], y[8];
        const typename Row8<T>::Raw held0 = raw0, held1 = raw1;
        Row8<T>::widen(raw0, x);
        Row8<T>::widen(raw1, y);
        if constexpr (NORM) {
            // (from the first pass that is all of q's rows on they stay the same)
            if (base == part * ROWS || base < n_k + n_v + splits * ROWS) {
                const float* w = is_k ? norm.k_weight : norm.q_weight;
                typename Row8<float>::Raw w0 = Row8<float>::load(w + a0), w1 = Row8<float>::load(w + a1);
                Row8<float>::widen(w0, wx);
                Row8<float>::widen(w1, wy);
            }
            if (!is_v) {
                const float by = row_norm<UNITS>(x, y, norm.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] = x[i] * by * wx[i];
                    y[i] = y[i] * by * wy[i];
                }
            }
        }
        if (turned) {
            if (rope.interleaved) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = x[2 * i], c = x[2 * i + 1], d = y[2 * i], e = y[2 * i + 1];
                    x[2 * i] = turned_a(a, c, cs[i]);
                    x[2 * i + 1] = turned_b(a, c, cs[i]);
                    y[2 * i] = turned_a(d, e, cs[4 + i]);
                    y[2 * i + 1] = turned_b(d, e, cs[4 + i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float a = x[i], c = y[i];
                    x[i] = turned_a(a, c, cs[i]);
                    y[i] = turned_b(a, c, cs[i]);
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
        } else if (CACHE == PLAIN && (is_k || is_v)) {
            if (valid && row0 >= 0) {
                T* dst = (T*)(is_k ? plain.k : plain.v) + (row0 + (long long)head * b.page_size) * D;
                if (is_k) {
                    Row8<T>::store(dst + a0, x);
                    Row8<T>::store(dst + a1, y);
                } else {
                    *(typename Row8<T>::Raw*)(dst + a0) = held0;     // bit for bit
                    *(typename Row8<T>::Raw*)(dst + a1) = held1;
                }
            }
        } else if (valid) {
            const int heads = is_k ? b.num_kv_heads : b.num_q_heads;
            T* dst = (T*)(is_k ? rows.k_out : rows.q_out) + ((long long)t * heads + head) * D;
            Row8<T>::store(dst + a0, x);
            Row8<T>::store(dst + a1, y);
        }
    }
}

template <typename T, int D, bool QUANT, bool ROPE>
__global__ __launch_bounds__(64 * WAVES) void rope_rows_kernel(BatchView b, RopeView rope, NewRows rows, Fp8Pools pools, Splits splits)
{
    do_rows<T, D, QUANT ? FP8 : NO_CACHE, ROPE, false>(b, rope, rows, pools, PlainPools{}, NormView{}, splits);
}

// With norms, a cache in the batch's dtype, or given slots
template <typename T, int D, int CACHE, bool ROPE, bool NORM>
__global__ __launch_bounds__(64 * WAVES) void norm_rope_rows_kernel(BatchView b, RopeView rope, NewRows rows, Fp8Pools pools, PlainPools plain,
                                                                    NormView norm, Splits splits)
{
    do_rows<T, D, CACHE, ROPE, NORM>(b, rope, rows, pools, plain, norm, splits);
}

// 16 codes to the batch's dtype, exact
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ inline void widen16(const u32x4 w, int byte, __bf16* dst)
{
    const float scale = up_scale(byte);
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
__device__ inline void widen16(const u32x4 w, int byte, float* dst)
{
    const float scale = up_scale(byte);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, true);
        *(float4*)(dst + 4 * i) = make_float4(lo[0], lo[1], hi[0], hi[1]);
    }
}

// Reads codes, writes 16 to 32 bits for each: bound by what it writes.  TOKENS: slots of a wave, whose rows travel together (four a wave
// 25.0 us where two take 24.4, stores past the caches 25.0).
template <typename T, int D, int TOKENS>
__global__ __launch_bounds__(64 * WAVES) void kv_gather_fp8_kernel(BatchView b, Fp8Pools pools, T* __restrict__ k_out, T* __restrict__ v_out)
{
    constexpr int UNITS = D / 16, ROWS = 64 / UNITS;
    const int t0 = (blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * TOKENS, lane = threadIdx.x & 63;
    if (t0 >= b.total_new_tokens) return;
    long long row0[TOKENS];
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) row0[i] = t0 + i < b.total_new_tokens ? pool_row(b, place_of_token(b, t0 + i)) : -1;
    const int u = lane % UNITS;
    for (int row = lane / UNITS; row < 2 * b.num_kv_heads; row += ROWS) {
        const bool is_k = row < b.num_kv_heads;
        const int head = is_k ? row : row - b.num_kv_heads;
        u32x4 codes[TOKENS];
        int byte[TOKENS];
#pragma unroll
        for (int i = 0; i < TOKENS; ++i) {
            const long long at = max(row0[i], 0ll) + (long long)head * b.page_size;
            const u32x4* from = (const u32x4*)((is_k ? pools.k : pools.v) + at * D + 16 * u);
            if constexpr (TOKENS > 1) codes[i] = __builtin_nontemporal_load(from);       // read once: other lines stay in the caches
            else codes[i] = *from;
            byte[i] = (is_k ? pools.k_scale : pools.v_scale)[at];
        }
#pragma unroll
        for (int i = 0; i < TOKENS; ++i)
            if (row0[i] >= 0) widen16(codes[i], byte[i], (is_k ? k_out : v_out) + ((long long)(t0 + i) * b.num_kv_heads + head) * D + 16 * u);
    }
}

// Few tokens: a wave for each pass over a token's rows, which takes its turns by itself; many: a wave for a token.
template <int D>
Splits splits_of(const BatchView& b, const NewRows& rows, bool cached, dim3& grid)
{
    const int heads = (rows.k != nullptr ? b.num_kv_heads : 0) + (cached ? b.num_kv_heads : 0) + (rows.q != nullptr ? b.num_q_heads : 0);
    const int passes = (heads * (D / 16) + 63) / 64;
    const int splits = (long long)b.total_new_tokens * passes <= MOST_SPLIT ? passes : 1;
    const long long items = (long long)b.total_new_tokens * splits;
    grid = dim3((unsigned)((items + WAVES - 1) / WAVES));
    return {splits, divisor_of(splits)};
}

template <typename T, int D>
hipError_t launch_rows(const BatchView& b, const RopeView& rope, const NewRows& rows, const Fp8Pools* pools, hipStream_t stream)
{
    dim3 grid;
    const dim3 block(64 * WAVES);
    const Splits splits = splits_of<D>(b, rows, pools != nullptr, grid);
    if (pools == nullptr) hipLaunchKernelGGL((rope_rows_kernel<T, D, false, true>), grid, block, 0, stream, b, rope, rows, Fp8Pools{}, splits);
    else if (rope.rotary_dim > 0) hipLaunchKernelGGL((rope_rows_kernel<T, D, true, true>), grid, block, 0, stream, b, rope, rows, *pools, splits);
    else hipLaunchKernelGGL((rope_rows_kernel<T, D, true, false>), grid, block, 0, stream, b, rope, rows, *pools, splits);
    return hipGetLastError();
}

template <typename T, int D, int CACHE>
hipError_t launch_norm_rows(const BatchView& b, const NormView& norm, const RopeView& rope, const NewRows& rows, const Fp8Pools& fp8, const PlainPools& plain,
                            hipStream_t stream)
{
    dim3 grid;
    const dim3 block(64 * WAVES);
    const Splits splits = splits_of<D>(b, rows, CACHE != NO_CACHE, grid);
    const bool turns = rope.rotary_dim > 0, norms = norm.q_weight != nullptr;
    if (turns && norms) hipLaunchKernelGGL((norm_rope_rows_kernel<T, D, CACHE, true, true>), grid, block, 0, stream, b, rope, rows, fp8, plain, norm, splits);
    else if (norms) hipLaunchKernelGGL((norm_rope_rows_kernel<T, D, CACHE, false, true>), grid, block, 0, stream, b, rope, rows, fp8, plain, norm, splits);
    else hipLaunchKernelGGL((norm_rope_rows_kernel<T, D, CACHE, true, false>), grid, block, 0, stream, b, rope, rows, fp8, plain, norm, splits);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_gather(const BatchView& b, const Fp8Pools& pools, void* k_out, void* v_out, hipStream_t stream)
{
    // A slot a wave where the caches can hold the call (12000 slots of 4 heads in bf16 10.0 us, and 11.6 the other way, 24000 16.3 and
    // 18.9), two with their loads past the caches where not (16384 of 8 heads 23.7 and 26.6, 35000 of 4 24.2 and 28.6).
    const long long bytes = 2ll * b.total_new_tokens * b.num_kv_heads * (D + 1 + D * (long long)sizeof(T));
    auto grid = [&](int tokens) { return dim3((unsigned)(((long long)b.total_new_tokens + WAVES * tokens - 1) / (WAVES * tokens))); };
    if (bytes < STREAM_BYTES)
        hipLaunchKernelGGL((kv_gather_fp8_kernel<T, D, 1>), grid(1), dim3(64 * WAVES), 0, stream, b, pools, (T*)k_out, (T*)v_out);
    else
        hipLaunchKernelGGL((kv_gather_fp8_kernel<T, D, 2>), grid(2), dim3(64 * WAVES), 0, stream, b, pools, (T*)k_out, (T*)v_out);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_rows(const BatchView& b, bool bf16, const RopeView& rope, const NewRows& rows, const Fp8Pools* pools, hipStream_t stream)
{
    if (bf16) return b.head_dim == 128 ? launch_rows<__bf16, 128>(b, rope, rows, pools, stream) : launch_rows<__bf16, 64>(b, rope, rows, pools, stream);
    return b.head_dim == 128 ? launch_rows<float, 128>(b, rope, rows, pools, stream) : launch_rows<float, 64>(b, rope, rows, pools, stream);
}

hipError_t launch_norm_rope_rows(const BatchView& b, bool bf16, const NormView& norm, const RopeView& rope, const NewRows& rows, const Fp8Pools* fp8,
                                 const PlainPools* plain, hipStream_t stream)
{
    auto go = [&](auto type, auto d) {
        typedef decltype(type) T;
        constexpr int D = decltype(d)::value;
        if (fp8 != nullptr) return launch_norm_rows<T, D, FP8>(b, norm, rope, rows, *fp8, PlainPools{}, stream);
        if (plain != nullptr) return launch_norm_rows<T, D, PLAIN>(b, norm, rope, rows, Fp8Pools{}, *plain, stream);
        return launch_norm_rows<T, D, NO_CACHE>(b, norm, rope, rows, Fp8Pools{}, PlainPools{}, stream);
    };
    using wide = std::integral_constant<int, 128>;
    using narrow = std::integral_constant<int, 64>;
    if (bf16) return b.head_dim == 128 ? go(__bf16{}, wide{}) : go(__bf16{}, narrow{});
    return b.head_dim == 128 ? go(float{}, wide{}) : go(float{}, narrow{});
}

hipError_t launch_kv_gather_fp8(const BatchView& b, bool bf16, const Fp8Pools& pools, void* k_out, void* v_out, hipStream_t stream)
{
    if (bf16) return b.head_dim == 128 ? launch_gather<__bf16, 128>(b, pools, k_out, v_out, stream) : launch_gather<__bf16, 64>(b, pools, k_out, v_out, stream);
    return b.head_dim == 128 ? launch_gather<float, 128>(b, pools, k_out, v_out, stream) : launch_gather<float, 64>(b, pools, k_out, v_out, stream);
}

}  // namespace emm
