// Attention of few rows over the 8-bit cache: decode steps and the shortest chunks (formulas: include/emm_fp8.h).
//
// Bound by reading K and V.  Rows are (new token, query head of a KV group) pairs of one (request, KV head), token-major; all of
// a pair's, 16 or 32 at most, are done together, so that each code is read once.
//
// Work is dealt by keys: the 32-key tiles of all pairs, request by request and head by head, are one line, which the
// workgroups share in equal parts whatever the lengths are; a workgroup finds its part by the sums of the lengths, which every
// wave takes by itself.  A part that is a whole pair is finished on the spot; of any other a workgroup leaves a record
// (sums, reference, unnormalised rows) of its first and of its last pair at most, and a second kernel adds the
// records of a pair up.  Inside a workgroup the four waves take a pair's tiles in turn, straight from global memory to
// registers, and meet in LDS at the end of the pair.
//
// Scores, S^T = K Q^T: v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 keys with all 128 channels as they lie in the cache, a
// key's scale byte beside them.  q is the sum of two 8-bit parts (split4); the second product carries the 1/16 in its
// block scale.
// Values, O^T += V^T P^T: v_mfma_f32_16x16x32_bf16 wants for each channel 8 keys of a lane side by side.  A lane reads 8
// neighbouring channels of the 8 keys whose scores it holds (the accumulators of two score products, which are then
// its part of the operand P^T as they are), pairs keys by byte permutes, and v_cvt_scalef32_pk_bf16_fp8 makes two bf16 of
// a pair.  V's scales go into P (a power of two).
#include <algorithm>

#include "attn_fp8_common.h"

namespace emm {

namespace {

using namespace fp8;

constexpr int D = HEAD_DIM;
constexpr int WAVES = 4;
constexpr int TILE = 32;                                 // keys per step of a wave
constexpr int ROWS = 16;
constexpr int LEAST_TILES = 4;                           // of a part: one for each wave
constexpr int WORKGROUPS = 1024;                         // four on each compute unit

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

// how the batch's tiles are dealt
struct RowsLayout {
    int G, workgroups, least;                            // least: tiles of a part
    Divisor by_G, by_kv_heads;
};

// a request's rows and keys, and where its tiles lie in the line (of one KV head; heads follow each other)
struct Request {
    int r, N, P, first_row;
    int tiles;                                           // per KV head
    long long before;                                    // tiles per KV head of the requests before it
};

// What the wave's lanes see of 64 requests at a time.  (A request without queries has no tiles; one with queries and no keys has
// one, with nothing to see in it, so that its rows are written.)
template <bool CAUSAL>
struct Line {
    const BatchView& b;
    int lane, N, P, cu, tiles, incl, first;
    long long total;

    __device__ int look(int from)                        // returns the tiles of the 64
    {
        const int r = min(from + lane, b.num_reqs - 1);
        const int n = b.new_lens[r], p = b.prefix_lens[r];
        cu = b.cu_new_lens[r];
        N = clamp_new_len(b, n, CAUSAL);
        P = clamp_prefix_len(b, p, CAUSAL ? N : 0);
        const int ctx = CAUSAL ? P + N : P;
        tiles = from + lane < b.num_reqs && N > 0 ? max((ctx + TILE - 1) / TILE, 1) : 0;
        incl = scan64(tiles);
        first = from;
        return __builtin_amdgcn_readlane(incl, 63);
    }
    __device__ explicit Line(const BatchView& batch) : b(batch), lane(threadIdx.x & 63), total(0)
    {
        for (int from = 0; from < b.num_reqs; from += 64) total += look(from);
    }
    __device__ Request take(int at, long long before_chunk) const
    {
        Request q;
        q.r = first + at;
        q.N = __builtin_amdgcn_readlane(N, at);
        q.P = __builtin_amdgcn_readlane(P, at);
        q.first_row = clamp_first_row(b, __builtin_amdgcn_readlane(cu, at), q.N);
        q.tiles = __builtin_amdgcn_readlane(tiles, at);
        q.before = before_chunk + __builtin_amdgcn_readlane(incl, at) - q.tiles;
        return q;
    }
    // the request that holds tile x of the line of one head, x < total
    __device__ Request holding(long long x)
    {
        long long before = 0;
        for (int from = 0;; from += 64) {
            const int sum = b.num_reqs <= 64 ? (int)total : look(from);
            if (x < before + sum || from + 64 >= b.num_reqs)
                return take(__builtin_ctzll(__builtin_amdgcn_ballot_w64(incl > (int)(x - before)) | 1ull << 63), before);
            before += sum;
        }
    }
    __device__ Request request(int r)
    {
        long long before = 0;
        for (int from = 0;; from += 64) {
            const int sum = b.num_reqs <= 64 ? (int)total : look(from);
            if (r < from + 64) return take(r - from, before);
            before += sum;
        }
    }
};

__device__ inline int part_tiles(const RowsLayout& L, long long all) { return (int)max((long long)L.least, (all + L.workgroups - 1) / L.workgroups); }

// A record: RT * 16 rows of 128 values, then (reference, sum) of each.  Workgroup w has two: of the pair its part begins in, of the pair
// that it ends in.
template <int RT> constexpr int RECORD_FLOATS = RT * ROWS * (D + 2);

template <bool CAUSAL, int RT>
__global__ __launch_bounds__(64 * WAVES) void attn_fp8_rows_kernel(AttnFp8Args a, RowsLayout L)
{
    const BatchView& b = a.b;
    __shared__ float part_o[WAVES][ROWS][D + 4];
    __shared__ float part_m[WAVES][ROWS], part_l[WAVES][ROWS];
    Line<CAUSAL> line(b);
    const long long all = line.total * b.num_kv_heads;
    const int share = part_tiles(L, all);
    long long x = (long long)blockIdx.x * share;
    const long long x_end = min(x + share, all);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int n16 = lane & 15, g = lane >> 4;
    const float c = b.softmax_scale * LOG2E;
    bool first_segment = true;
    while (x < x_end) {
        const Request rq = line.holding(x / b.num_kv_heads);
        const long long off = x - rq.before * b.num_kv_heads;
        if (off < 0 || off >= (long long)rq.tiles * b.num_kv_heads) return;      // (lengths that change meanwhile)
        const int kvh = (int)(off / rq.tiles), t0 = (int)(off - (long long)kvh * rq.tiles);
        const int t1 = (int)min((long long)rq.tiles, t0 + (x_end - x));
        x += t1 - t0;
        const int n_rows = min(rq.N * L.G, RT * ROWS);
        const int ctx = CAUSAL ? rq.P + rq.N : rq.P;                     // slots that hold tokens
        const int all_see = CAUSAL ? rq.P + 1 : rq.P;                    // keys that every row sees
        const int last_block = max(((ctx + 15) >> 4) - 1, 0);

        QParts q[RT];
        int limit[RT];                                                   // last key that the lane's row sees
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int row = min(rt * ROWS + n16, n_rows - 1), tok = L.by_G.quotient(row);
            limit[rt] = CAUSAL ? rq.P + tok : rq.P - 1;
            const __bf16* qp = (const __bf16*)a.q + ((long long)(rq.first_row + tok) * b.num_q_heads + kvh * L.G + row - tok * L.G) * D;
            // channels 16 g .. + 15 and 64 + 16 g .. + 15, of q and of K alike
            bf16x8 qv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) qv[i] = *(const bf16x8*)(qp + 64 * (i >> 1) + 16 * g + 8 * (i & 1));
            q[rt] = split_q(qv);
        }
        const int32_t* __restrict__ pt = b.page_table + (long long)rq.r * b.max_pages;
        float m[RT], l[RT];
        f32x4 o[RT][8];                                                  // channels 32 g + 8 v + i of the row, in o[i][v]
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -INFINITY;
            l[rt] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[rt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        // lane 2 j + k: block k of the wave's j-th tile from `ids_from` on, in 16-key blocks of the pool
        int ids = 0;
        auto ask_ids = [&](int from) {
            const int blk = min(2 * (from + WAVES * (lane >> 1)) + (lane & 1), last_block);
            const int page = min(max(pt[blk >> b.page_shift], 0), b.num_pages - 1);
            ids = ((page * b.num_kv_heads + kvh) << b.page_shift) + (blk & ((1 << b.page_shift) - 1));
        };
        int nth = 0;
        for (int t = t0 + wave; t < t1; t += WAVES, ++nth) {
            if ((nth & 31) == 0) ask_ids(t);
            uint4 kc[4];
            uint2 v[8];
            uint32_t vs[2];
            int ks[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const long long at = (long long)__builtin_amdgcn_readlane(ids, 2 * (nth & 31) + k) * 16;     // row of the pool
                const unsigned char* kp = a.pools.k + at * D + n16 * D + 16 * g;
                kc[2 * k] = *(const uint4*)kp;
                kc[2 * k + 1] = *(const uint4*)(kp + 64);
                ks[k] = (a.pools.k_scale + at)[n16];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[4 * k + i] = *(const uint2*)(a.pools.v + at * D + (4 * g + i) * D + 8 * n16);
                vs[k] = *(const uint32_t*)(a.pools.v_scale + at + 4 * g);
            }
            f32x4 s[RT][2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const i32x8 kf = {(int)kc[2 * k].x, (int)kc[2 * k].y, (int)kc[2 * k].z, (int)kc[2 * k].w, (int)kc[2 * k + 1].x, (int)kc[2 * k + 1].y, (int)kc[2 * k + 1].z,
                                  (int)kc[2 * k + 1].w};
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    s[rt][k] = f32x4{0.f, 0.f, 0.f, 0.f};
                    s[rt][k] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, q[rt].high, s[rt][k], 0, 0, 0, ks[k], 0, q[rt].scale_high);
                    s[rt][k] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, q[rt].low, s[rt][k], 0, 0, 0, ks[k], 0, q[rt].scale_low);
                }
            }
            const int key0 = t * TILE + 4 * g;                           // key of score (k, i): key0 + 16 k + i
            const bool masked = (t + 1) * TILE > all_see;
            uint32_t nans = 0;
            if (masked) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = key0 + 16 * k + i;
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt)
                            if (key > limit[rt]) s[rt][k][i] = -INFINITY;
                        if (key >= ctx) {                                // whatever lies there must not meet a weight of zero
                            v[4 * k + i] = make_uint2(0, 0);
                            vs[k] = (vs[k] & ~(0xffu << (8 * i))) | (uint32_t)BIAS << (8 * i);
                        }
                        nans |= nan_bytes(v[4 * k + i].x) | nan_bytes(v[4 * k + i].y);
                    }
            }
            bf16x8 p[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float top = fmaxf(fmaxf(fmaxf(s[rt][0][0], s[rt][0][1]), fmaxf(s[rt][0][2], s[rt][0][3])),
                                  fmaxf(fmaxf(s[rt][1][0], s[rt][1][1]), fmaxf(s[rt][1][2], s[rt][1][3])));
                top = row_max(top) * c;
                if (__builtin_amdgcn_ballot_w64(top > m[rt]) != 0) {
                    const float to = fmaxf(m[rt], top);
                    const float scale = to > m[rt] ? __builtin_amdgcn_exp2f(m[rt] - to) : 1.0f;     // (m is -inf at first: 0)
                    m[rt] = to;
                    l[rt] *= scale;
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[rt][i] *= scale;
                }
                const float ref = m[rt] == -INFINITY ? 0.f : m[rt];      // a row that has seen no key yet
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float w = __builtin_amdgcn_exp2f(fmaf(s[rt][k][i], c, -ref));
                        l[rt] += w;
                        p[rt][4 * k + i] = (__bf16)(w * up_scale(vs[k] >> (8 * i) & 0xff));
                    }
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
            auto values = [&](int i, bf16x8 vf) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) o[rt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[rt], o[rt][i], 0, 0, 0);
            };
            if (masked && __builtin_amdgcn_ballot_w64(nans != 0) != 0) {
                // A NaN in V of a key that only some of the rows see: a weight of zero does not keep it out.  It is taken out, and the rows
                // that see such a key get it afterwards, by a product of which is what.
                uint2 marks[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t nx = nan_bytes(v[i].x) >> 7, ny = nan_bytes(v[i].y) >> 7;    // 1 in each byte that is a NaN
                    marks[i] = make_uint2(nx * 0x38u, ny * 0x38u);                              // the code of 1.0
                    v[i] = make_uint2(v[i].x & ~(nx * 0xffu), v[i].y & ~(ny * 0xffu));
                }
                product(values);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[k] = marks[k];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) p[rt][k] = key0 + 16 * (k >> 2) + (k & 3) <= limit[rt] ? (__bf16)1.0f : (__bf16)0.0f;
                }
                product([&](int i, bf16x8 vf) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[rt], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (hit[k] > 0.f) o[rt][i][k] = __builtin_nanf("");
                    }
                });
            } else {
                product(values);
            }
        }
        // the waves' parts of 16 rows at a time, 8 channels of a row per thread
        const bool whole = t0 == 0 && t1 == rq.tiles;
        float* rec = (float*)a.workspace + (2ll * blockIdx.x + (first_segment ? 0 : 1)) * RECORD_FLOATS<RT>;
        first_segment = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (rt * ROWS >= n_rows) break;                              // (the same for all waves)
            __syncthreads();
            const float l_row = row_sum(l[rt]);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) part_o[wave][n16][32 * g + 8 * k + i] = o[rt][i][k];
            if (g == 0) {
                part_m[wave][n16] = m[rt];
                part_l[wave][n16] = l_row;
            }
            __syncthreads();
            const int in_rows = threadIdx.x >> 4, ch = (threadIdx.x & 15) * 8, row = rt * ROWS + in_rows;
            if (row >= n_rows) continue;
            float top = -INFINITY, sum = 0.f, acc[8] = {};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) top = fmaxf(top, part_m[w][in_rows]);
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(part_m[w][in_rows] - ref);
                sum = fmaf(part_l[w][in_rows], f, sum);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] = fmaf(part_o[w][in_rows][ch + i], f, acc[i]);
            }
            if (!whole) {
                *(f32x4*)(rec + row * D + ch) = f32x4{acc[0], acc[1], acc[2], acc[3]};
                *(f32x4*)(rec + row * D + ch + 4) = f32x4{acc[4], acc[5], acc[6], acc[7]};
                if ((threadIdx.x & 15) == 0) *(f32x2*)(rec + RT * ROWS * D + 2 * row) = f32x2{top, sum};
                continue;
            }
            const int tok = L.by_G.quotient(row);
            const long long dst = (long long)(rq.first_row + tok) * b.num_q_heads + kvh * L.G + row - tok * L.G;
            const float inv = sum == 0.f ? 0.f : 1.0f / sum;             // no key at all: a row of zeros
            bf16x8 res;
#pragma unroll
            for (int i = 0; i < 8; ++i) res[i] = (__bf16)(acc[i] * inv);
            *(bf16x8*)((__bf16*)a.out + dst * D + ch) = res;
            if (a.lse != nullptr && (threadIdx.x & 15) == 0) a.lse[dst] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
        }
    }
}

// The records of a row of a pair that several workgroups had parts of.  Half a wave takes a record at a time, 4 channels a lane.
template <bool CAUSAL, int RT>
__global__ __launch_bounds__(64 * WAVES) void attn_fp8_merge_rows_kernel(AttnFp8Args a, RowsLayout L, int rows_most)
{
    const BatchView& b = a.b;
    const int row = blockIdx.x % rows_most, pair = blockIdx.x / rows_most;
    const int r = L.by_kv_heads.quotient(pair), kvh = pair - r * b.num_kv_heads;
    Line<CAUSAL> line(b);
    const long long all = line.total * b.num_kv_heads;
    const int share = part_tiles(L, all);
    const Request rq = line.request(r);
    if (row >= rq.N * L.G || rq.tiles == 0) return;
    const long long x = rq.before * b.num_kv_heads + (long long)kvh * rq.tiles;
    const int w0 = (int)(x / share), w1 = (int)((x + rq.tiles - 1) / share);
    if (w0 == w1) return;                                                // done where it was
    __shared__ float part[2 * WAVES][D + 4];
    __shared__ float part_l[2 * WAVES];
    const int lane = threadIdx.x & 63, half = threadIdx.x >> 5, ch = (threadIdx.x & 31) * 4;
    // the first workgroup's record is its last pair's, unless the pair is where its part begins; of the others it is the first
    auto record = [&](int w) { return (const float*)a.workspace + (2ll * w + (w == w0 && x != (long long)w0 * share ? 1 : 0)) * RECORD_FLOATS<RT>; };
    float top = -INFINITY;
    for (int w = w0 + lane; w <= w1; w += 64) top = fmaxf(top, record(w)[RT * ROWS * D + 2 * row]);
#pragma unroll
    for (int i = 1; i < 64; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
    const float ref = top == -INFINITY ? 0.f : top;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll 4
    for (int w = w0 + half; w <= w1; w += 2 * WAVES) {
        const float* rec = record(w);
        const f32x4 v = *(const f32x4*)(rec + row * D + ch);
        const f32x2 ml = *(const f32x2*)(rec + RT * ROWS * D + 2 * row);
        const float f = __builtin_amdgcn_exp2f(ml[0] - ref);
        sum = fmaf(ml[1], f, sum);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = fmaf(v[i], f, acc[i]);
    }
    *(f32x4*)&part[half][ch] = acc;
    if ((threadIdx.x & 31) == 0) part_l[half] = sum;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    sum = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2 * WAVES; ++i) {
        sum += part_l[i];
        acc += *(const f32x4*)&part[i][ch];
    }
    const int tok = L.by_G.quotient(row);
    const long long dst = (long long)(rq.first_row + tok) * b.num_q_heads + kvh * L.G + row - tok * L.G;
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 res;
#pragma unroll
    for (int i = 0; i < 4; ++i) res[i] = (__bf16)(acc[i] * inv);
    *(bf16x4*)((__bf16*)a.out + dst * D + ch) = res;
    if (a.lse != nullptr && threadIdx.x == 0) a.lse[dst] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
}

constexpr int MOST_ROWS = 2 * ROWS;
long long rows_of(const BatchView& b) { return (long long)b.max_new_len * (b.num_q_heads / b.num_kv_heads); }

RowsLayout layout_of(const BatchView& b)
{
    RowsLayout L;
    L.G = b.num_q_heads / b.num_kv_heads;
    L.by_G = divisor_of(L.G);
    L.by_kv_heads = divisor_of(b.num_kv_heads);
    L.least = LEAST_TILES;
    // no more workgroups than the page table can hold work for
    const long long tiles = ((long long)b.max_pages * b.page_size + TILE - 1) / TILE, all = tiles * b.num_reqs * b.num_kv_heads;
    L.workgroups = (int)std::min<long long>(WORKGROUPS, (all + L.least - 1) / L.least);
    return L;
}
size_t rows_workspace_bytes(const BatchView& b) { return 2 * (size_t)layout_of(b).workgroups * (rows_of(b) <= ROWS ? RECORD_FLOATS<1> : RECORD_FLOATS<2>) * sizeof(float); }

template <bool CAUSAL, int RT>
hipError_t launch_rows(const AttnFp8Args& a, hipStream_t stream)
{
    const RowsLayout L = layout_of(a.b);
    const int rows = (int)rows_of(a.b);
    hipLaunchKernelGGL((attn_fp8_rows_kernel<CAUSAL, RT>), dim3(L.workgroups), dim3(64 * WAVES), 0, stream, a, L);
    if (L.workgroups > 1)
        hipLaunchKernelGGL((attn_fp8_merge_rows_kernel<CAUSAL, RT>), dim3((unsigned)a.b.num_reqs * a.b.num_kv_heads * rows), dim3(64 * WAVES), 0, stream, a, L, rows);
    return hipGetLastError();
}

}  // namespace

// Few rows of a (request, KV head): their keys are split over the chip.  Many: rows over the waves, keys through LDS.
size_t attn_fp8_workspace_bytes(const BatchView& b)
{
    if (b.num_reqs == 0 || b.total_new_tokens == 0) return 0;
    return rows_of(b) <= MOST_ROWS ? rows_workspace_bytes(b) : attn_fp8_tiles_workspace_bytes(b);
}

hipError_t launch_attn_fp8(const AttnFp8Args& a, bool causal, hipStream_t stream)
{
    if (rows_of(a.b) > MOST_ROWS) return launch_attn_fp8_tiles(a, causal, stream);
    if (rows_of(a.b) <= ROWS) return causal ? launch_rows<true, 1>(a, stream) : launch_rows<false, 1>(a, stream);
    return causal ? launch_rows<true, 2>(a, stream) : launch_rows<false, 2>(a, stream);
}

}  // namespace emm
