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
// Small calls are bound by the trips through memory that follow each other, and finding the part is one of them.  Where the page table says
// that they are small, every pair has the same number of workgroups, which share its own tiles: nobody sums the lengths of others, the
// merge's records travel with the lengths, and where the table holds no more than 512 tokens there is one part and no merge.
//
// Scores, S^T = K Q^T: a lane has 32 channels of a key, which v_cvt_scalef32_pk_bf16_fp8 makes bf16 in the key's scale (exact)
// for four v_mfma_f32_16x16x32_bf16, and the same 32 channels of its row of q.
// Values, O^T += V^T P^T: v_mfma_f32_16x16x32_bf16 wants for each channel 8 keys of a lane side by side.  A lane reads 8
// neighbouring channels of the 8 keys whose scores it holds (the accumulators of two score products, which are then
// its part of the operand P^T as they are), pairs keys by byte permutes, and v_cvt_scalef32_pk_bf16_fp8 makes two bf16 of
// a pair.  V's scales go into P (a power of two; a weight is rounded to bf16 after it, half a step off either way.  With V's least
// scale, 2^-117, weights below 2^-9 of the row's largest are subnormal there, and off by up to 2^-17 of it.)
// Weights are rounded to bf16 because the product takes both operands so; in 32 bits it would need 16 times the matrix instructions.
// out is then 0.0018 of itself off (root mean square) where its own rounding makes 0.0017.
//
// Measured (28 query heads over 4 KV heads unless said): 64 contexts of 8192 96 us with the records' merge, 5.6 TB/s of the cache's
// bytes, 91 without it; 32 contexts of 300 to 4600 with 32 over 8 heads 41.5 us, 4.1 TB/s (a request with little to do at its end
// has its record, its merge and its start like any other: 36 us of the main kernel, of which 26 are bytes).  In fixed parts, under tables as wide
// as the contexts, calls in a graph: one of 1500 7.4 us, of which an empty launch after the other would be 3.4 (called one by one 7.5 in some runs
// and 8.5 in others), one of 60 4.4, 32 of 200 6.0, 8 of 2000 10.5, one of 16000 12.4; what wider tables cost stands at FIXED_TILES.
#include <algorithm>
#include <type_traits>

#include "attn_fp8_common.h"

namespace emm {

namespace {

using namespace fp8;

constexpr int D = HEAD_DIM;
constexpr int WAVES = 4;                                 // of a workgroup; a compute unit holds two
constexpr int SUMS = 8 / WAVES;
constexpr int TILE = 32;                                 // keys per step of a wave
constexpr int ROWS = 16;
constexpr int OUT_STRIDE = D + 8;                        // bf16 values between output rows in LDS
constexpr int LEAST_TILES = WAVES;                       // of a part: one for each wave
// Fixed parts, where the page table holds at most so many tiles for each of the workgroups; as a line in brackets, us.  Tables as wide as the
// longest context: 16 of 300 to 8000 23.8 (25.6), 32 of 2000 19.3 (22.2), one of 1500 7.4 (11.0), of the next size, 48 of 400 to 4000, 39.7
// (33.2).  Wider ones: one of 1500 with room for 8 k, 32 k, 128 k tokens 9.1, 10.0, 9.9 (12.0); one of 500 8.9, 9.8, 9.9 (9.0); 16 of 1500 with room
// for 8 k 12.6 (15.6), of the next size, for 32 k, 12.6 (15.5).  (Parts by the table's width, whatever the contexts are: one of 1500 9.9, 11.6,
// 20.8; 16 of 1500 22.1.)
constexpr int FIXED_TILES = 32;
constexpr int WHOLE_TILES = 16;                          // in the table, for a pair that one workgroup does (32 of 500 9.3 us, in parts of four 11.4; of twice the pairs
                                                         // 11.1 and 15.2; one of 1000, which would be 10.6, has parts: 7.5)
constexpr int WORKGROUPS = 512;                          // two on each compute unit (256 of twice the waves: ragged 49 us in place of 42)
constexpr int ALONE = 256;                               // so many parts have a compute unit to themselves
constexpr int MANY_RECORDS = 16;                         // of a pair: then 1024 threads merge (one of 16000 14.4 us, and 16.5 with 256; ragged 41.9, 48.2 with 1024)
constexpr int STREAM_TILES = 12000;                      // 96 MiB of codes: from here on a call does not fit the last-level cache next to others, and its
                                                         // loads go past the caches (64 of 8192 96 us, and 103 through them; 32 of 2000 21.4, 22.7 past them)
constexpr int MOST_COMPARED = 512;                       // requests among which shared pages are looked for

// of the four lanes (l, l ^ 16, l ^ 32, l ^ 48) that hold a row
__device__ inline float row_max(float x) { return pair_max(max16(x)); }
__device__ inline float row_sum(float x) { return pair_sum(sum16(x)); }

// how the batch's tiles are dealt
struct RowsLayout {
    int G, workgroups;
    int parts;                                           // fixed: workgroups of a pair; else 0
    Divisor by_G, by_kv_heads, by_workgroups, by_parts;
};

// a request's rows and keys, and where its tiles lie in the line (of one KV head; heads follow each other)
struct Request {
    int r, N, P, first_row;
    int tiles;                                           // per KV head
    int before;                                          // tiles per KV head of the requests before it
};

// What the wave's lanes see of 64 requests at a time.  (A request without queries has no tiles; one with queries and no keys has
// one, with nothing to see in it, so that its rows are written.)
template <bool CAUSAL>
struct Line {
    const BatchView& b;
    int lane, N, P, cu, tiles, incl, first;
    int total;                                           // (the whole line is below 2^31 tiles: see launch_attn_fp8)

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
    __device__ Request take(int at, int before_chunk) const
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
    __device__ Request holding(int x)
    {
        int before = 0;
        for (int from = 0;; from += 64) {
            const int sum = b.num_reqs <= 64 ? total : look(from);
            if (x < before + sum || from + 64 >= b.num_reqs)
                return take(__builtin_ctzll(__builtin_amdgcn_ballot_w64(incl > x - before) | 1ull << 63), before);
            before += sum;
        }
    }
    __device__ Request request(int r)
    {
        int before = 0;
        for (int from = 0;; from += 64) {
            const int sum = b.num_reqs <= 64 ? total : look(from);
            if (r < from + 64) return take(r - from, before);
            before += sum;
        }
    }
};

// Tiles of a part of the line: equal shares for all workgroups, but not too short ones.  (Parts of four tiles where each has a compute unit to itself,
// of eight at least else: as a line, one context of 1500 tokens 11.4 us with 4 and 12.4 with 8, 8 of 2000 15.0 and 13.6, one of 16000 17.6 and 15.0.)
__device__ inline int part_tiles(const RowsLayout& L, int all)
{
    return max(all <= LEAST_TILES * ALONE ? LEAST_TILES : 2 * LEAST_TILES, L.by_workgroups.quotient(all - 1) + 1);
}
// Tiles of a fixed part of a pair that has so many in all, where it may have several.  (Short parts only where a merge has few of them: one of
// 16000 12.0 us in parts of 8 tiles, and 13.8 of 4; of 1500 8.7 and 7.5.)
__host__ __device__ inline int least_fixed_part(long long tiles) { return tiles <= MANY_RECORDS * LEAST_TILES ? LEAST_TILES : 2 * LEAST_TILES; }
__device__ inline int fixed_part(const RowsLayout& L, int tiles)
{
    return L.parts == 1 ? tiles : max(least_fixed_part(tiles), L.by_parts.quotient(tiles + L.parts - 1));
}
// x / d, the same in all lanes, for d > 0, 0 <= x < 2^31 and a quotient below 2^20: by the reciprocal, which is off by less than one whole
__device__ inline int small_quotient(int x, int d)
{
    const int q = __builtin_amdgcn_readfirstlane((int)((float)x * __builtin_amdgcn_rcpf((float)d)));
    const int rest = x - q * d;
    return rest < 0 ? q - 1 : rest >= d ? q + 1 : q;
}

// a fixed deal's request
template <bool CAUSAL>
__device__ inline Request request_of(const BatchView& b, int r)
{
    int n = b.new_lens[r], p = b.prefix_lens[r], cu = b.cu_new_lens[r];
    n = __builtin_amdgcn_readfirstlane(n), p = __builtin_amdgcn_readfirstlane(p), cu = __builtin_amdgcn_readfirstlane(cu);
    asm volatile("" : "+s"(n), "+s"(p), "+s"(cu));                       // one trip for the three
    Request q;
    q.r = r;
    q.N = clamp_new_len(b, n, CAUSAL);
    q.P = clamp_prefix_len(b, p, CAUSAL ? q.N : 0);
    q.first_row = clamp_first_row(b, cu, q.N);
    q.tiles = q.N > 0 ? max(((CAUSAL ? q.P + q.N : q.P) + TILE - 1) / TILE, 1) : 0;
    q.before = 0;
    return q;
}

// a row's place among the packed (token, head) rows
__device__ inline long long place_of(const BatchView& b, const RowsLayout& L, const Request& rq, int kvh, int row)
{
    const int tok = L.by_G.quotient(row);
    return (long long)(rq.first_row + tok) * b.num_q_heads + kvh * L.G + row - tok * L.G;
}

// A record: RT * 16 rows of 128 values in the order of the accumulators, then (reference, sum) of each.  Workgroup w has two: of the pair its part begins in, of the pair
// that it ends in.
template <int RT> constexpr int RECORD_FLOATS = RT * ROWS * (D + 2);

// 16 bytes or 8 of a row of codes, with the non-temporal hint or without
template <class T, bool STREAM>
__device__ inline T fetch(const unsigned char* base, uint32_t offset)
{
    typedef uint32_t V __attribute__((ext_vector_type(sizeof(T) / 4)));
    const V* p = (const V*)(base + offset);
    if constexpr (STREAM) return __builtin_bit_cast(T, __builtin_nontemporal_load(p));
    else return __builtin_bit_cast(T, *p);
}

// a part of a pair: the pair's tiles t0 .. t1 - 1
struct Segment {
    Request rq;
    int kvh, t0, t1, n_rows, ctx;
};

struct NoLine { int total; };                            // in its place where parts are fixed

template <bool CAUSAL, int RT, bool FIXED>
__global__ __launch_bounds__(64 * WAVES, 2) void attn_fp8_rows_kernel(AttnFp8Args a, RowsLayout L)
{
    const BatchView& b = a.b;
    __shared__ f32x4 part_o[WAVES][ROWS * D / 4];
    __shared__ f32x2 part_ml[WAVES][ROWS];
    auto line = [&] { if constexpr (FIXED) return NoLine{1}; else return Line<CAUSAL>(b); }();
    const int all = line.total * b.num_kv_heads;
    if (all == 0) return;
    const int share = FIXED ? 0 : part_tiles(L, all);
    int x = FIXED ? 0 : (int)min((long long)blockIdx.x * share, (long long)all);
    const int x_end = FIXED ? 1 : x + min(share, all - x);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int n16 = lane & 15, g = lane >> 4;
    const float c = b.softmax_scale * LOG2E;

    // the segment that begins at x; x moves behind it.  t1 == t0: none.
    auto next_segment = [&]() -> Segment {
        Segment s = {};
        if (x >= x_end) return s;
        if constexpr (FIXED) {
            const int pair = L.by_parts.quotient(blockIdx.x), r = L.by_kv_heads.quotient(pair);
            s.rq = request_of<CAUSAL>(b, r);
            s.kvh = pair - r * b.num_kv_heads;
            const int size = fixed_part(L, s.rq.tiles);
            s.t0 = min((int)(blockIdx.x - pair * L.parts) * size, s.rq.tiles);
            s.t1 = min(s.t0 + size, s.rq.tiles);
            x = x_end;
        } else {
            s.rq = line.holding(L.by_kv_heads.quotient(x));
            const int off = x - s.rq.before * b.num_kv_heads;
            if (off < 0 || s.rq.tiles <= 0) return s;                    // (lengths that change meanwhile)
            s.kvh = min(small_quotient(off, s.rq.tiles), b.num_kv_heads - 1);
            s.t0 = off - s.kvh * s.rq.tiles;
            s.t1 = max(min(s.rq.tiles, s.t0 + (x_end - x)), s.t0);
            x += s.t1 - s.t0;
        }
        s.n_rows = min(s.rq.N * L.G, RT * ROWS);
        s.ctx = CAUSAL ? s.rq.P + s.rq.N : s.rq.P;                       // slots that hold tokens
        return s;
    };
    // lane 2 j + k: block k of the wave's j-th tile from `from` on, in 16-key blocks of the pool
    auto ask_ids = [&](const Segment& s, int from) -> int {
        const int blk = min(2 * (from + WAVES * (lane >> 1)) + (lane & 1), max(((s.ctx + 15) >> 4) - 1, 0));
        const int page = min(max(b.page_table[(long long)s.rq.r * b.max_pages + (blk >> b.page_shift)], 0), b.num_pages - 1);
        return ((page * b.num_kv_heads + s.kvh) << b.page_shift) + (blk & ((1 << b.page_shift) - 1));
    };
    // Are K and V of the segment to go past the caches?  Not where all of a call fits them, nor where another request holds the same
    // pages: what the first brings in serves the others.
    auto streamed = [&](const Segment& s) -> bool {
        if (FIXED || all < STREAM_TILES || s.t0 >= s.t1) return false;
        const int entry = min((2 * s.t0) >> b.page_shift, b.max_pages - 1);
        const int mine = b.page_table[(long long)s.rq.r * b.max_pages + entry];
        bool shared = false;
        for (int from = 0; from < min(b.num_reqs, MOST_COMPARED); from += 64) {
            const int r = min(from + lane, b.num_reqs - 1);
            shared |= r != s.rq.r && b.page_table[(long long)r * b.max_pages + entry] == mine;
        }
        return __builtin_amdgcn_ballot_w64(shared) == 0;
    };
    // q's rows: channels 16 g .. + 15 and 64 + 16 g .. + 15, of q and of K alike
    auto ask_q = [&](const Segment& s, int rt, uint32_t (&pairs)[16]) {
        const __bf16* qp = (const __bf16*)a.q + place_of(b, L, s.rq, s.kvh, min(rt * ROWS + n16, s.n_rows - 1)) * D;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 w = *(const uint4*)(qp + 64 * (i >> 1) + 16 * g + 8 * (i & 1));
            pairs[4 * i] = w.x; pairs[4 * i + 1] = w.y; pairs[4 * i + 2] = w.z; pairs[4 * i + 3] = w.w;
        }
    };
    struct Tile {
        uint4 k[4];
        uint2 v[8];                                                      // of key 4 g + i of block 0, then of block 1: channels 8 n16 .. + 7
        uint32_t v_scale[2];
        int k_scale[2];
    };
    const uint32_t k_at = n16 * D + 16 * g, v_at = 4 * g * D + 8 * n16;
    auto load_as = [&](int ids, int nth, auto streamed, Tile& to) {
        constexpr bool STREAM = decltype(streamed)::value;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const long long at = (long long)__builtin_amdgcn_readlane(ids, 2 * (nth & 31) + k) * 16;     // row of the pool
            const unsigned char *kp = a.pools.k + at * D, *vp = a.pools.v + at * D;
            to.k[2 * k] = fetch<uint4, STREAM>(kp, k_at);
            to.k[2 * k + 1] = fetch<uint4, STREAM>(kp, k_at + 64);
            to.k_scale[k] = (a.pools.k_scale + at)[(uint32_t)n16];
#pragma unroll
            for (int i = 0; i < 4; ++i) to.v[4 * k + i] = fetch<uint2, STREAM>(vp, v_at + i * D);
            to.v_scale[k] = *(const uint32_t*)(a.pools.v_scale + at + (uint32_t)(4 * g));
        }
    };
    auto load = [&](int ids, int nth, bool stream, Tile& to) {
        if (stream) {
            asm volatile("" ::: "memory");                               // (the two ways are one load without a hint to the optimiser otherwise)
            load_as(ids, nth, std::true_type{}, to);
            asm volatile("" ::: "memory");
        } else {
            load_as(ids, nth, std::false_type{}, to);
        }
    };

    constexpr bool AHEAD = RT == 1;                                      // one tile is computed, one travels (32 rows leave no registers for that)
    Tile even, odd;
    Segment now = next_segment();
    if (now.t0 >= now.t1) return;
    int ids = ask_ids(now, now.t0 + wave);
    uint32_t pairs[RT][16];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) ask_q(now, rt, pairs[rt]);
    bool stream = streamed(now);
    if (AHEAD && now.t0 + wave < now.t1) load(ids, 0, stream, even);
    for (bool first_segment = true;; first_segment = false) {
        const int all_see = CAUSAL ? now.rq.P + 1 : now.rq.P;            // keys that every row sees
        int limit[RT];                                                   // last key that the lane's row sees
        bf16x8 q[RT][4];                                                 // of the lane's row: the channels that it has of a key
        float m[RT], l[RT];
        f32x4 o[RT][8];                                                  // channels 32 g + 8 v + i of the row, in o[i][v]
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            limit[rt] = CAUSAL ? now.rq.P + L.by_G.quotient(min(rt * ROWS + n16, now.n_rows - 1)) : now.rq.P - 1;
#pragma unroll
            for (int j = 0; j < 4; ++j) q[rt][j] = __builtin_bit_cast(bf16x8, u32x4{pairs[rt][4 * j], pairs[rt][4 * j + 1], pairs[rt][4 * j + 2], pairs[rt][4 * j + 3]});
            m[rt] = -INFINITY;
            l[rt] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[rt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        // what the next segment begins with travels over this one's tiles
        const Segment then = next_segment();
        const bool more = then.t0 < then.t1;
        int then_ids = 0;
        if (more) {
            then_ids = ask_ids(then, then.t0 + wave);
            if (AHEAD) ask_q(then, 0, pairs[0]);
        }

        auto compute = [&](int t, Tile& tile) {
            uint2 (&v)[8] = tile.v;
            uint32_t (&vs)[2] = tile.v_scale;
            f32x4 s[RT][2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t codes[8] = {tile.k[2 * k].x, tile.k[2 * k].y, tile.k[2 * k].z, tile.k[2 * k].w, tile.k[2 * k + 1].x, tile.k[2 * k + 1].y,
                                           tile.k[2 * k + 1].z, tile.k[2 * k + 1].w};
                const float scale = up_scale(tile.k_scale[k]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) s[rt][k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    u32x4 w;                                             // 8 channels of the lane's key
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        w[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * j + i], scale, false));
                        w[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * j + i], scale, true));
                    }
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
                        s[rt][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), q[rt][j], s[rt][k], 0, 0, 0);
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
                        if (key >= now.ctx) {                            // whatever lies there must not meet a weight of zero
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
            bf16x8 sees[RT];
            uint2 marks[8];
            const bool some_nan = masked && __builtin_amdgcn_ballot_w64(nans != 0) != 0;
            if (some_nan) {
                // A NaN in V of a key that only some of the rows see: a weight of zero does not keep it out.  It is taken out, and the rows
                // that see such a key get it afterwards, by a product of which is what.
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t nx = nan_bytes(v[i].x) >> 7, ny = nan_bytes(v[i].y) >> 7;    // 1 in each byte that is a NaN
                    marks[i] = make_uint2(nx * 0x38u, ny * 0x38u);                              // the code of 1.0
                    v[i] = make_uint2(v[i].x & ~(nx * 0xffu), v[i].y & ~(ny * 0xffu));
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) sees[rt][i] = key0 + 16 * (i >> 2) + (i & 3) <= limit[rt] ? (__bf16)1.0f : (__bf16)0.0f;
                }
            }
            product([&](int i, bf16x8 vf) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) o[rt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[rt], o[rt][i], 0, 0, 0);
            });
            if (some_nan) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = marks[i];
                product([&](int i, bf16x8 vf) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, sees[rt], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (hit[k] > 0.f) o[rt][i][k] = __builtin_nanf("");
                    }
                });
            }
        };
        int nth = 0;
        auto step = [&](int t, Tile& tile, Tile& next) {                 // tile t; the one after it is asked for first
            if (t + WAVES < now.t1) {
                ++nth;
                if ((nth & 31) == 0) ids = ask_ids(now, t + WAVES);
                load(ids, nth, stream, next);
            }
            compute(t, tile);
        };
        if constexpr (AHEAD) {
            for (int t = now.t0 + wave; t < now.t1; t += 2 * WAVES) {
                step(t, even, odd);
                if (t + WAVES < now.t1) step(t + WAVES, odd, even);
            }
        } else {
            for (int t = now.t0 + wave; t < now.t1; t += WAVES, ++nth) {
                if (nth > 0 && (nth & 31) == 0) ids = ask_ids(now, t);
                load(ids, nth, stream, even);
                compute(t, even);
            }
        }
        if (more) {
            ids = then_ids;
            stream = streamed(then);
            if (AHEAD && then.t0 + wave < then.t1) load(ids, 0, stream, even);
        }

        // The waves' parts, 16 rows at a time, in the order of the accumulators: four of them, channels 32 g + 8 k + i for k = 0 .. 3, are
        // the 16 bytes at place i * 64 + lane.  A thread adds up SUMS places, its own and those that far behind.
        const bool whole = now.t0 == 0 && now.t1 == now.rq.tiles;
        float* rec = (float*)a.workspace + (FIXED ? (long long)blockIdx.x : 2ll * blockIdx.x + (first_segment ? 0 : 1)) * RECORD_FLOATS<RT>;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (rt * ROWS >= now.n_rows) break;                          // (the same for all waves)
            __syncthreads();
            const float l_row = row_sum(l[rt]);
#pragma unroll
            for (int i = 0; i < 8; ++i) part_o[wave][i * 64 + lane] = o[rt][i];
            if (g == 0) part_ml[wave][n16] = f32x2{m[rt], l_row};
            __syncthreads();
            float top = -INFINITY, sum = 0.f;
            f32x2 ml[WAVES];
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                ml[w] = part_ml[w][n16];
                top = fmaxf(top, ml[w][0]);
            }
            const float ref = top == -INFINITY ? 0.f : top;
            f32x4 acc[SUMS] = {};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(ml[w][0] - ref);
                sum = fmaf(ml[w][1], f, sum);
#pragma unroll
                for (int h = 0; h < SUMS; ++h) {
                    const f32x4 part = part_o[w][threadIdx.x + 64 * WAVES * h];
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[h][k] = fmaf(part[k], f, acc[h][k]);
                }
            }
            if (!whole) {
#pragma unroll
                for (int h = 0; h < SUMS; ++h) *(f32x4*)(rec + (rt * 512 + threadIdx.x + 64 * WAVES * h) * 4) = acc[h];
                if (threadIdx.x < ROWS) *(f32x2*)(rec + RT * ROWS * D + 2 * (rt * ROWS + threadIdx.x)) = f32x2{top, sum};
                continue;
            }
            // finished: rows in order again, through LDS
            const float inv = sum == 0.f ? 0.f : 1.0f / sum;             // no key at all: a row of zeros
            __syncthreads();
            __bf16* rows = (__bf16*)part_o;                              // [16][OUT_STRIDE]
#pragma unroll
            for (int h = 0; h < SUMS; ++h)
#pragma unroll
                for (int k = 0; k < 4; ++k) rows[n16 * OUT_STRIDE + 32 * g + 8 * k + wave + WAVES * h] = (__bf16)(acc[h][k] * inv);
            __syncthreads();
            const int out_row = threadIdx.x >> 4;
            if (threadIdx.x < 16 * ROWS && rt * ROWS + out_row < now.n_rows)
                *(uint4*)((__bf16*)a.out + place_of(b, L, now.rq, now.kvh, rt * ROWS + out_row) * D + 8 * n16) = *(const uint4*)(rows + out_row * OUT_STRIDE + 8 * n16);
            if (a.lse != nullptr && threadIdx.x < ROWS && rt * ROWS + n16 < now.n_rows)
                a.lse[place_of(b, L, now.rq, now.kvh, rt * ROWS + n16)] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
        }
        if (!more) return;
        if (!AHEAD) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) ask_q(then, rt, pairs[rt]);
        }
        now = then;
    }
}

// The records of a pair that several workgroups had parts of: a workgroup for 32 channels (a lane group of the records) of 16 rows,
// 128 threads of it a record at a time.  4 to 5 us, of which 1.7 are any launch's and 1.5 the lengths.  (The last workgroup of a pair
// merging in the first kernel saves that where parts are long and costs two trips through memory where they are not: 64 of 8192 94 us,
// but one of 1500 16, ragged 45.)
template <bool CAUSAL, int RT, int THREADS, bool FIXED>
__global__ __launch_bounds__(THREADS) void attn_fp8_merge_rows_kernel(AttnFp8Args a, RowsLayout L)
{
    constexpr int TEAMS = THREADS / 128, AT_ONCE = 8;
    const BatchView& b = a.b;
    const int g = blockIdx.x & 3, rt = RT == 1 ? 0 : (blockIdx.x >> 2) & 1, pair = blockIdx.x >> (RT == 1 ? 2 : 3);
    const int r = L.by_kv_heads.quotient(pair), kvh = pair - r * b.num_kv_heads;
    const int team = threadIdx.x >> 7, in_team = threadIdx.x & 127, i = in_team >> 4, n16 = threadIdx.x & 15;
    const int ml_at = RT * ROWS * D + 2 * (rt * ROWS + n16), v_at = (rt * 512 + i * 64 + 16 * g + n16) * 4;
    f32x4 v[AT_ONCE];
    f32x2 ml[AT_ONCE];
    auto fetch_record = [&](int u, long long at) {
        const float* rec = (const float*)a.workspace + at * RECORD_FLOATS<RT>;
        v[u] = *(const f32x4*)(rec + v_at);
        ml[u] = *(const f32x2*)(rec + ml_at);
    };
    if constexpr (FIXED) {                                               // the first of the records that there could be travel with the lengths
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) fetch_record(u, (long long)pair * L.parts + min(team + TEAMS * u, L.parts - 1));
        asm volatile("" ::: "memory");
    }
    Request rq;
    int w0, w1, odd = 0;                                                 // odd: the pair begins inside w0's part
    if constexpr (FIXED) {
        rq = request_of<CAUSAL>(b, r);
        w0 = pair * L.parts;
        w1 = w0 + small_quotient(max(rq.tiles - 1, 0), fixed_part(L, rq.tiles));
    } else {
        Line<CAUSAL> line(b);
        const int all = line.total * b.num_kv_heads;
        if (all == 0) return;
        const int share = part_tiles(L, all);
        rq = line.request(r);
        const int x = rq.before * b.num_kv_heads + kvh * rq.tiles;
        w0 = small_quotient(x, share);
        w1 = small_quotient(x + rq.tiles - 1, share);
        odd = x != w0 * share ? 1 : 0;
    }
    const int n_rows = min(rq.N * L.G, RT * ROWS);
    if (rt * ROWS >= n_rows || rq.tiles == 0 || w0 == w1) return;        // (one: done where it was)
    __shared__ f32x4 part[TEAMS][128];
    __shared__ f32x2 part_ml[TEAMS][ROWS];
    __shared__ __bf16 rows[ROWS][40];
    // the first workgroup's record is its last pair's, unless the pair is where its part begins; of the others it is the first
    auto record = [&](int w) { return FIXED ? (long long)w : 2ll * w + (w == w0 ? odd : 0); };
    float top = -INFINITY, sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    // what there is in terms of a larger reference, and more of it
    auto raise = [&](float to) -> float {
        const float ref = to == -INFINITY ? 0.f : to, f = __builtin_amdgcn_exp2f(top - ref);
        top = to;
        sum *= f;
        acc *= f;
        return ref;
    };
    auto take = [&](f32x4 v, float ref, f32x2 ml) {
        const float f = __builtin_amdgcn_exp2f(ml[0] - ref);
        sum = fmaf(ml[1], f, sum);
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] = fmaf(v[k], f, acc[k]);
    };
    for (int from = w0 + team; from <= w1; from += TEAMS * AT_ONCE) {
        if (!FIXED || from != w0 + team)
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) fetch_record(u, record(min(from + TEAMS * u, w1)));
        float most = top;
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
            if (from + TEAMS * u <= w1) most = fmaxf(most, ml[u][0]);
        const float ref = raise(most);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
            if (from + TEAMS * u <= w1) take(v[u], ref, ml[u]);
    }
    if (team > 0) {
        part[team][in_team] = acc;
        if (i == 0) part_ml[team][n16] = f32x2{top, sum};
    }
    __syncthreads();
    if (team == 0) {
        float most = top;
#pragma unroll
        for (int w = 1; w < TEAMS; ++w) most = fmaxf(most, part_ml[w][n16][0]);
        const float ref = raise(most);
#pragma unroll
        for (int w = 1; w < TEAMS; ++w) take(part[w][in_team], ref, part_ml[w][n16]);
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
        for (int k = 0; k < 4; ++k) rows[n16][8 * k + i] = (__bf16)(acc[k] * inv);
        if (a.lse != nullptr && g == 0 && i == 0 && rt * ROWS + n16 < n_rows)
            a.lse[place_of(b, L, rq, kvh, rt * ROWS + n16)] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
    }
    __syncthreads();
    const int out_row = threadIdx.x >> 2, at = 8 * (threadIdx.x & 3);
    if (threadIdx.x < 64 && rt * ROWS + out_row < n_rows)
        *(uint4*)((__bf16*)a.out + place_of(b, L, rq, kvh, rt * ROWS + out_row) * D + 32 * g + at) = *(const uint4*)&rows[out_row][at];
}

long long rows_of(const BatchView& b) { return (long long)b.max_new_len * (b.num_q_heads / b.num_kv_heads); }
// tiles that the page table could hold
long long line_of(const BatchView& b) { return ((long long)b.max_pages * b.page_size + TILE - 1) / TILE * b.num_reqs * b.num_kv_heads; }

RowsLayout layout_of(const BatchView& b)
{
    RowsLayout L;
    L.G = b.num_q_heads / b.num_kv_heads;
    L.by_G = divisor_of(L.G);
    L.by_kv_heads = divisor_of(b.num_kv_heads);
    // no more workgroups than the page table can hold work for
    L.workgroups = (int)std::max<long long>(std::min<long long>(WORKGROUPS, (line_of(b) + LEAST_TILES - 1) / LEAST_TILES), 1);
    L.parts = 0;
    const long long pairs = (long long)b.num_reqs * b.num_kv_heads, most = line_of(b) / pairs;    // tiles of a pair
    if (rows_of(b) <= ROWS && pairs <= WORKGROUPS && line_of(b) <= (long long)WORKGROUPS * FIXED_TILES) {
        const long long per_pair = WORKGROUPS / pairs;                   // workgroups that a pair may have
        const long long least = most <= WHOLE_TILES ? WHOLE_TILES : least_fixed_part(most);
        const long long part = std::max(least, (most + per_pair - 1) / per_pair);    // of a context that fills the table
        L.parts = (int)std::max<long long>((most + part - 1) / part, 1);
        L.workgroups = (int)pairs * L.parts;
    }
    L.by_parts = divisor_of(std::max(L.parts, 1));
    L.by_workgroups = divisor_of(L.workgroups);
    return L;
}
size_t rows_workspace_bytes(const BatchView& b)
{
    const RowsLayout L = layout_of(b);
    return (L.parts == 1 ? 0 : L.parts > 0 ? 1 : 2) * (size_t)L.workgroups * (rows_of(b) <= ROWS ? RECORD_FLOATS<1> : RECORD_FLOATS<2>) * sizeof(float);
}

template <bool CAUSAL, int RT, bool FIXED>
hipError_t launch_rows(const AttnFp8Args& a, const RowsLayout& L, hipStream_t stream)
{
    hipLaunchKernelGGL((attn_fp8_rows_kernel<CAUSAL, RT, FIXED>), dim3(L.workgroups), dim3(64 * WAVES), 0, stream, a, L);
    // few pairs have many records each: more of them at a time
    const long long pairs = (long long)a.b.num_reqs * a.b.num_kv_heads;
    const dim3 grid((unsigned)(pairs * 4 * RT));
    if (L.workgroups > MANY_RECORDS * pairs) hipLaunchKernelGGL((attn_fp8_merge_rows_kernel<CAUSAL, RT, 1024, FIXED>), grid, dim3(1024), 0, stream, a, L);
    else if (FIXED ? L.parts > 1 : L.workgroups > 1) hipLaunchKernelGGL((attn_fp8_merge_rows_kernel<CAUSAL, RT, 256, FIXED>), grid, dim3(256), 0, stream, a, L);
    return hipGetLastError();
}
template <bool CAUSAL>
hipError_t launch_few(const AttnFp8Args& a, hipStream_t stream)
{
    const RowsLayout L = layout_of(a.b);
    if (rows_of(a.b) > ROWS) return launch_rows<CAUSAL, 2, false>(a, L, stream);
    return L.parts > 0 ? launch_rows<CAUSAL, 1, true>(a, L, stream) : launch_rows<CAUSAL, 1, false>(a, L, stream);
}

}  // namespace

// Few rows of a (request, KV head): their keys are split over the chip.  Many: rows over the waves, keys through LDS; and 17 to 32
// rows of few pairs, which leave this kernel's two accumulators without a tile on the way (28 rows: 4 pairs of 1500 keys 11.0 us and
// 14.2 here, 16 pairs 12.9 and 15.2, of 16000 28.0 and 26.9; 32 pairs of 16000 44.5 and 38.7, 256 of 8000 137 and 113).
// (Tables so wide that the line could pass 2^31 tiles, a terabyte of cache or pages shared by thousands, go the second way.)
namespace {
constexpr int FEW_PAIRS = 16;
bool few_rows(const BatchView& b)
{
    return rows_of(b) <= ((long long)b.num_reqs * b.num_kv_heads > FEW_PAIRS ? 2 * ROWS : ROWS) && line_of(b) < (1ll << 31) - (1 << 20);
}
}  // namespace

size_t attn_fp8_workspace_bytes(const BatchView& b)
{
    if (b.num_reqs == 0 || b.total_new_tokens == 0) return 0;
    return few_rows(b) ? rows_workspace_bytes(b) : attn_fp8_tiles_workspace_bytes(b);
}

hipError_t launch_attn_fp8(const AttnFp8Args& a, bool causal, hipStream_t stream)
{
    if (!few_rows(a.b)) return launch_attn_fp8_tiles(a, causal, stream);
    return causal ? launch_few<true>(a, stream) : launch_few<false>(a, stream);
}

}  // namespace emm
