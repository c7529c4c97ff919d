// Attention over the 8-bit cache (formulas: include/emm_fp8.h).
//
// Rows are (new token, query head of a KV group) pairs of one (request, KV head), token-major.  A workgroup takes 16 of
// them, its four waves take the keys 32 at a time, in turn, straight from global memory to registers, and meet in LDS
// at the end.
//
// Scores, S^T = K Q^T: v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 keys with all 128 channels as they lie in the cache, a
// key's scale byte beside them.  q is the sum of two 8-bit parts, high = nearest e4m3 of q 2^-e and low = 16 (q 2^-e - high),
// exact for a bf16 down to 2^-22 of its row's largest (four significant bits each); the second product carries the 1/16
// in its block scale.
// Values, O^T += V^T P^T: v_mfma_f32_16x16x32_bf16 wants for each channel 8 keys of a lane side by side.  A lane reads 8
// neighbouring channels of the 8 keys whose scores it holds (the accumulators of two score products, which are then
// its part of the operand P^T as they are), pairs keys by byte permutes, and v_cvt_scalef32_pk_bf16_fp8 makes two bf16 of
// a pair.  V's scales go into P (a power of two).
#include "attn_fp8_common.h"

namespace emm {

namespace {

using namespace fp8;

constexpr int D = HEAD_DIM;
constexpr int WAVES = 4;
constexpr int TILE = 32;                                 // keys per step of a wave
constexpr int ROWS = 16;

// largest of the four lanes (l, l ^ 16, l ^ 32, l ^ 48) that hold a row
__device__ inline float row_max(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float row_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// q's operands of the score product: 32 channels of the lane's row
struct QParts {
    i32x8 high, low;
    int scale_high, scale_low;                           // scale bytes
};
__device__ inline QParts split_q(const bf16x8 (&q)[4])
{
    float x[32];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        x[i] = (float)q[i >> 3][i & 7];
        most = max(most, finite(x[i]) ? __float_as_uint(x[i]) & 0x7fffffffu : 0u);
    }
    most = max(most, (uint32_t)__shfl_xor((int)most, 16));
    most = max(most, (uint32_t)__shfl_xor((int)most, 32));
    QParts p;
    p.scale_high = scale_byte(most);
    p.scale_low = p.scale_high + LOW_PART_SCALE;
    const float down = down_scale(p.scale_high);
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        const float part[4] = {x[4 * w], x[4 * w + 1], x[4 * w + 2], x[4 * w + 3]};
        const QCodes c = split4(part, down);
        p.high[w] = (int)c.high;
        p.low[w] = (int)c.low;
    }
    return p;
}

template <bool CAUSAL>
__global__ __launch_bounds__(64 * WAVES) void attn_fp8_rows_kernel(AttnFp8Args a)
{
    const BatchView& b = a.b;
    __shared__ float part_o[WAVES][ROWS][D + 4];
    __shared__ float part_m[WAVES][ROWS], part_l[WAVES][ROWS];
    const int r = blockIdx.z, kvh = blockIdx.y;
    const int G = b.num_q_heads / b.num_kv_heads;
    const int N = clamp_new_len(b, b.new_lens[r], CAUSAL);
    const int n_rows = N * G, row0 = blockIdx.x * ROWS;
    if (row0 >= n_rows) return;
    const int P = clamp_prefix_len(b, b.prefix_lens[r], CAUSAL ? N : 0);
    const int first_row = clamp_first_row(b, b.cu_new_lens[r], N);
    const int ctx = CAUSAL ? P + N : P;                                  // slots that hold tokens
    const int kv_len = CAUSAL ? P + (min(row0 + ROWS, n_rows) - 1) / G + 1 : P;   // keys that these rows see
    const int all_see = CAUSAL ? P + row0 / G + 1 : P;                   // keys that every one of them sees
    const int n_blocks = (ctx + 15) >> 4;
    const int n_tiles = (kv_len + TILE - 1) / TILE;

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int n16 = lane & 15, g = lane >> 4;
    const int row = min(row0 + n16, n_rows - 1), tok = row / G;
    const int limit = CAUSAL ? P + tok : P - 1;                          // last key that the lane's row sees
    const __bf16* qp = (const __bf16*)a.q + ((long long)(first_row + tok) * b.num_q_heads + kvh * G + row - tok * G) * D;
    // channels 16 g .. + 15 and 64 + 16 g .. + 15, of q and of K alike
    bf16x8 qv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) qv[i] = *(const bf16x8*)(qp + 64 * (i >> 1) + 16 * g + 8 * (i & 1));
    const QParts q = split_q(qv);

    const int32_t* __restrict__ pt = b.page_table + (long long)r * b.max_pages;
    const float c = b.softmax_scale * LOG2E;
    float m = -INFINITY, l = 0.f;
    f32x4 o[8] = {};                                                     // channels 32 g + 8 v + i of the row, in o[i][v]
    for (int t = wave; t < n_tiles; t += WAVES) {
        // where the two 16-key blocks lie, in rows of the pool
        long long at[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int blk = min(2 * t + k, n_blocks - 1);
            const int page = min(max(pt[blk >> b.page_shift], 0), b.num_pages - 1);
            at[k] = ((((long long)page * b.num_kv_heads + kvh) << b.page_shift) + (blk & ((1 << b.page_shift) - 1))) * 16;
        }
        f32x4 s[2];
        uint2 v[8];
        uint32_t vs[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const unsigned char* kp = a.pools.k + (at[k] + n16) * D + 16 * g;
            const uint4 k0 = *(const uint4*)kp, k1 = *(const uint4*)(kp + 64);
            const int ks = a.pools.k_scale[at[k] + n16];
            const i32x8 kf = {(int)k0.x, (int)k0.y, (int)k0.z, (int)k0.w, (int)k1.x, (int)k1.y, (int)k1.z, (int)k1.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * k + i] = *(const uint2*)(a.pools.v + (at[k] + 4 * g + i) * D + 8 * n16);
            vs[k] = *(const uint32_t*)(a.pools.v_scale + at[k] + 4 * g);
            s[k] = f32x4{0.f, 0.f, 0.f, 0.f};
            s[k] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, q.high, s[k], 0, 0, 0, ks, 0, q.scale_high);
            s[k] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, q.low, s[k], 0, 0, 0, ks, 0, q.scale_low);
        }
        const int key0 = t * TILE + 4 * g;                               // key of score (k, i): key0 + 16 k + i
        const bool masked = (t + 1) * TILE > all_see;
        uint32_t nans = 0;
        if (masked) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = key0 + 16 * k + i;
                    if (key > limit) s[k][i] = -INFINITY;
                    if (key >= ctx) {                                    // whatever lies there must not meet a weight of zero
                        v[4 * k + i] = make_uint2(0, 0);
                        vs[k] = (vs[k] & ~(0xffu << (8 * i))) | (uint32_t)BIAS << (8 * i);
                    }
                    nans |= nan_bytes(v[4 * k + i].x) | nan_bytes(v[4 * k + i].y);
                }
        }
        float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        top = row_max(top) * c;
        if (__builtin_amdgcn_ballot_w64(top > m) != 0) {
            const float to = fmaxf(m, top);
            const float scale = to > m ? __builtin_amdgcn_exp2f(m - to) : 1.0f;     // (m is -inf at first: 0)
            m = to;
            l *= scale;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] *= scale;
        }
        const float ref = m == -INFINITY ? 0.f : m;                      // a row that has seen no key yet
        bf16x8 p;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = __builtin_amdgcn_exp2f(fmaf(s[k][i], c, -ref));
                l += w;
                p[4 * k + i] = (__bf16)(w * up_scale(vs[k] >> (8 * i) & 0xff));
            }
        // V's operands: pairs of keys (j, j + 1), channels by bytes
        auto product = [&](auto&& add) {
            uint32_t pair[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                pair[j][0] = __builtin_amdgcn_perm(v[2 * j + 1].x, v[2 * j].x, 0x05010400u);
                pair[j][1] = __builtin_amdgcn_perm(v[2 * j + 1].x, v[2 * j].x, 0x07030602u);
                pair[j][2] = __builtin_amdgcn_perm(v[2 * j + 1].y, v[2 * j].y, 0x05010400u);
                pair[j][3] = __builtin_amdgcn_perm(v[2 * j + 1].y, v[2 * j].y, 0x07030602u);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                u32x4 w;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = __builtin_bit_cast(uint32_t, (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(pair[j][i >> 1], 1.0f, true)
                                                               : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(pair[j][i >> 1], 1.0f, false));
                add(i, __builtin_bit_cast(bf16x8, w));
            }
        };
        if (masked && __builtin_amdgcn_ballot_w64(nans != 0) != 0) {
            // A NaN in V of a key that only some of the rows see: a weight of zero does not keep it out.  It is taken out, and the rows
            // that see such a key get it afterwards, by a product of which is what.
            uint2 marks[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t x = nan_bytes(v[i].x) >> 7, y = nan_bytes(v[i].y) >> 7;      // 1 in each byte that is a NaN
                marks[i] = make_uint2(x * 0x38u, y * 0x38u);                                // the code of 1.0
                v[i] = make_uint2(v[i].x & ~(x * 0xffu), v[i].y & ~(y * 0xffu));
            }
            product([&](int i, bf16x8 vf) { o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p, o[i], 0, 0, 0); });
            bf16x8 sees;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                sees[k] = key0 + 16 * (k >> 2) + (k & 3) <= limit ? (__bf16)1.0f : (__bf16)0.0f;
                v[k] = marks[k];
            }
            product([&](int i, bf16x8 vf) {
                const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, sees, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (hit[k] > 0.f) o[i][k] = __builtin_nanf("");
            });
        } else {
            product([&](int i, bf16x8 vf) { o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p, o[i], 0, 0, 0); });
        }
    }
    l = row_sum(l);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) part_o[wave][n16][32 * g + 8 * k + i] = o[i][k];
    if (g == 0) {
        part_m[wave][n16] = m;
        part_l[wave][n16] = l;
    }
    __syncthreads();
    // the waves' parts, 8 channels of a row per thread
    const int out_row = threadIdx.x >> 4, ch = (threadIdx.x & 15) * 8;
    if (row0 + out_row >= n_rows) return;
    float top = -INFINITY, sum = 0.f, acc[8] = {};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, part_m[w][out_row]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(part_m[w][out_row] - ref);
        sum = fmaf(part_l[w][out_row], f, sum);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = fmaf(part_o[w][out_row][ch + i], f, acc[i]);
    }
    const int out_tok = (row0 + out_row) / G, head = kvh * G + row0 + out_row - out_tok * G;
    const long long dst = (long long)(first_row + out_tok) * b.num_q_heads + head;
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;                     // no key at all: a row of zeros
    bf16x8 res;
#pragma unroll
    for (int i = 0; i < 8; ++i) res[i] = (__bf16)(acc[i] * inv);
    *(bf16x8*)((__bf16*)a.out + dst * D + ch) = res;
    if (a.lse != nullptr && (threadIdx.x & 15) == 0) a.lse[dst] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
}

}  // namespace

// Few rows of a (request, KV head): their keys are split over the waves.  Many: rows over the waves, keys through LDS.
namespace {
bool few_rows(const BatchView& b) { return (long long)b.max_new_len * (b.num_q_heads / b.num_kv_heads) <= ROWS; }
}  // namespace

size_t attn_fp8_workspace_bytes(const BatchView& b) { return few_rows(b) ? 0 : attn_fp8_tiles_workspace_bytes(b); }

hipError_t launch_attn_fp8(const AttnFp8Args& a, bool causal, hipStream_t stream)
{
    if (!few_rows(a.b)) return launch_attn_fp8_tiles(a, causal, stream);
    const int G = a.b.num_q_heads / a.b.num_kv_heads;
    const dim3 grid((unsigned)(((long long)a.b.max_new_len * G + ROWS - 1) / ROWS), (unsigned)a.b.num_kv_heads, (unsigned)a.b.num_reqs);
    if (causal) hipLaunchKernelGGL(attn_fp8_rows_kernel<true>, grid, dim3(64 * WAVES), 0, stream, a);
    else hipLaunchKernelGGL(attn_fp8_rows_kernel<false>, grid, dim3(64 * WAVES), 0, stream, a);
    return hipGetLastError();
}

}  // namespace emm
