// Attention with a window and sinks over the paged bf16 cache, head_dim 128 (include/emm_step.h says which slots a row sees).
//
// A row is one (new token j, query head g of a KV group), index j * G + g, so that the G heads that share a KV head are neighbours.
// The rows of a tile look at slots from the first that its first row's window holds to its last row's own, and at the sinks before
// them.  In blocks of 16 slots, which lie in one page each, these are a list without a gap: the sinks' blocks, then the window's.
// Tiles are taken from that list, so nothing is fetched or multiplied that no row sees, but for the ends of blocks and tiles.
//
// Shapes:
//   rows    a workgroup of 4 or 8 waves has 32 rows a wave, and its waves share tiles of 64 keys: prompts, bound by the matrix pipes and the
//           power that they take.  How its row tiles are dealt, cut and halved stands at RowsPlan.
//   decode  one new token, up to 16 heads: a workgroup has a (request, KV head), each of its four waves takes every fourth tile of 32 keys by
//           itself, without a barrier, and they meet in LDS at the end.  Bound by reading K and V.
//   keys    the same with 32 rows a wave: chunks too small for the rows shape, bound by the trips through memory that follow each other.
// Where the last two are too few to fill the chip their keys are cut into parts besides, and a second kernel adds the parts' records up.
// K and V go from memory straight into LDS, whole rows of 256 bytes in XOR-swizzled chunks of 16; K is read with ds_read_b128, V with
// the transposing read.  Scores are made transposed, S^T = K Q^T, and K's rows are stored with bits 2 and 3 of the place in the block
// swapped: then a lane has one row's scores, and those are the value product's operand O^T += V^T P^T as they stand.
//
// The softmax's reference is a row's maximum of an earlier tile: it is raised, and the sums scaled, only when a tile brings a score that
// is more than 2^LAG of it, which the lane's own maximum tells without asking the other half of the row.  (Any reference gives the same
// quotient; weights are at most 2^LAG.)  Weights are rounded to bf16 because the product takes both operands so; their sum is of what they were
// before, in 32 bits, so that lse is as exact as the scores (of the rounded ones it could be off by their half step, 2^-8).
//
// A slot that some row of a tile sees and another does not may hold an infinity or NaN, which a weight of 0 would not remove.  In the
// tiles at the ends of windows such values are looked for, replaced by 0, and added at the end to the rows that see them.
//
// Measured, 28 query heads over 4 KV heads, calls in a graph: 2 x 2048 new tokens behind a window of 4096 232 to 244 us by card (990 to 1040 TFLOP/s of what rows
// see, where matrix products of 8192 and 16384 reach 1265 and 1375: 448 units on 256 compute units, two waves to a SIMD, matrix pipes busy half of the cycles at 1.95 GHz;
// from rest the clock dips, and calls in a row take 250, then up to 312, and settle after about a hundred); one compute unit's fill of units, 2 x 1170, 135 us;
// 8 x 177 to 479 behind 1024 62 to 66 us; 36 tokens behind 2048 13.4; one decode step behind 1024 7.7 (two launches; the kernels 4.4 and 3.1 traced); 64 behind 4096
// 83 us (6.5 TB/s), behind 1024 24.
#include "attn_bf16_common.h"
#include "step_internal.h"

#include <algorithm>
#include <type_traits>

namespace emm {

namespace {

using namespace bf16attn;

constexpr int WAVES = 4;                                 // of a workgroup of the keys shape
constexpr int WAVE_ROWS = 32;
constexpr int BLK = 16;                                  // slots of a block
constexpr int SLAB = BLK * D * 2;                        // bytes of a block of one KV head
constexpr int OUT_STRIDE = 272;                          // bytes between output rows in LDS
constexpr int REC_STRIDE = D + 4;                        // floats between rows of records, in LDS and in the workspace: D values, m, l
constexpr float LAG = 16.0f;                             // log2 of the largest weight
constexpr float LN2 = 0.69314718055994530942f, LOG2E = 1.44269504088896340736f;

struct WindowLayout {
    int G;
    Divisor by_G, by_kv_heads;
    // rows shape
    int most_parts;                                      // into how many parts the units of an XCD's last round may be cut: see RowsPlan
    // keys shape
    int slots;                                           // row tiles per KV head that the grid has room for
    int single;                                          // 1: a request has one row tile at most, and slot r is request r's
    int parts;                                           // of a row tile's keys
    int per_xcd;                                         // items of an XCD, in order; 0: item i is workgroup i
    int items;
    Divisor by_slots, by_parts;
};

// A row tile: which request's, and the list of blocks that its rows look at
struct Tile {
    int r, N, P, first_row;                              // request, new tokens, cached tokens, packed row of the first new token
    int row0, n_rows;                                    // first row; rows of the (request, KV head)
    int last;                                            // the last slot that any row sees
    int low_first, low_last;                             // first slot of the first row's window, of the last row's
    int sink_blocks, gap, blocks;                        // the list: blocks 0 .. sink_blocks - 1, then the others `gap` further on
    __device__ int block(int v) const { return v + (v >= sink_blocks ? gap : 0); }
};

// How a row tile's keys are cut where the host has given it `parts` workgroups, from what a window may hold: each takes `share` of its tiles, so many at least
// as are worth a workgroup, so that a context shorter than its window has fewer parts, and the others nothing to do and no record.
// MIN_TILES: of a part: of the decode shape one of 32 keys for each wave, of the rows shape of 64.  us with 2, 4, 8, 16: one decode step behind 1024 8.7, 8.0, 8.8,
// 10.4, behind 4096 10.0, 9.8, 9.8, 10.6; 250 tokens behind 1024 20.1, 20.0, 22.9, 21.9; 2 x 200 behind 4096 43.5, 43.2, 43.3, 45.9.
constexpr int MIN_TILES = 4;
constexpr int MIN_TILES_KEYS = 1;                        // (20 tokens of 320 11.7 us, in parts of four 13.3)
__device__ inline int share_of(int tiles, int parts, const Divisor& by_parts, int least) { return max(by_parts.quotient(tiles + parts - 1), least); }
__device__ inline int share_of(int tiles, int parts) { return max((tiles + parts - 1) / parts, MIN_TILES); }

// The tile of `rows` rows from row0 on of a request with these lengths; false: it has no such rows.
__device__ inline bool make_tile(const BatchView& b, const WindowLayout& L, const WindowView& w, int r, long long row0, int rows, int new_len,
                                 int prefix_len, int cu, Tile& t)
{
    t.r = r;
    t.N = clamp_new_len(b, new_len, true);
    t.n_rows = t.N * L.G;                                // (at most 2^30: see check_rows)
    if (row0 < 0 || row0 >= t.n_rows) return false;
    t.row0 = (int)row0;
    t.P = clamp_prefix_len(b, prefix_len, t.N);
    t.first_row = clamp_first_row(b, cu, t.N);
    t.last = t.P + L.by_G.quotient(min(t.row0 + rows, t.n_rows) - 1);
    t.low_first = window_low(w, t.P + L.by_G.quotient(t.row0));
    t.low_last = window_low(w, t.last);
    const int first_block = t.low_first / BLK;
    t.sink_blocks = min((int)(((uint32_t)w.sinks + BLK - 1) / BLK), first_block);
    t.gap = first_block - t.sink_blocks;
    t.blocks = t.last / BLK + 1 - t.gap;
    return true;
}

// ---- Keys shape: slots.  First row tile of request r: its ceil(rows / ROWS) tiles fit between this and the next request's, whatever cu_new_lens[r] is.
template <int ROWS> __device__ inline long long first_slot(int cu_new, int G, int r) { return (long long)max(cu_new, 0) * G / ROWS + r; }

// The tile in `slot`; false: there is none.  Uniform over the workgroup.
template <int ROWS> __device__ inline bool find_tile(const BatchView& b, const WindowLayout& L, const WindowView& w, int slot, Tile& t)
{
    int r = slot;
    if (!L.single) {
        int lo = 0, hi = b.num_reqs;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first_slot<ROWS>(b.cu_new_lens[mid], L.G, mid) <= slot) lo = mid; else hi = mid;
        }
        r = lo;
    }
    const int new_len = b.new_lens[r], prefix_len = b.prefix_lens[r], cu = b.cu_new_lens[r];
    const long long row0 = L.single ? 0 : ((long long)slot - first_slot<ROWS>(cu, L.G, r)) * ROWS;
    return make_tile(b, L, w, r, row0, ROWS, new_len, prefix_len, cu, t);
}

// ---- Rows shape, NW waves a workgroup.  A unit is a row tile of 32 NW rows of a KV head; units are counted head by head, request by request, and
// each XCD has an eighth of them, neighbours, which mostly read the same keys.  It holds 256 / NW workgroups at once, and units take about equally
// long (a window), so that with few units in the last round most of its places would idle.  Such units are
//   cut     along their keys into as many parts as there are places for, which leave records for a second kernel, or, where that gains nothing,
//   halved  a workgroup then has half of the rows, two waves to 32 of them, which take a half of each tile's keys each and meet in LDS.
// Everybody derives the same plan from the lengths.
// Four waves, two workgroups to a compute unit, whose starts and ends overlap, for short windows (8 x 177 to 479 tokens behind 1024 62 us, and 70 with eight);
// eight, which bring each tile once for twice the rows, for long ones (2 x 2048 behind 4096 240 us, and 251 with four).
// us whole, halved, cut, of units that are left over on an XCD (the more parts there are, the more their records cost, 67 or 135 KB each, out and in):
//   eight waves, behind 4096: 3 units 92, 62, 31; 8 95, 67, 51; 10 (3 parts) 96, 70, 60; 13 (2) 97, 75, 76; 16 (2) 100, 84, 83; behind 32 others: 5 219, 199, 170; 13
//     224, 207, 204.  So they are cut from two parts on.
//   four waves, behind 1024: 5 units 25, 22, 18.6; 8 (4 parts) 25, 22, 20.5; 10 (3) 24.8, 22.6, 22.8; 13 (2) 25, 23, 26; 16 (2) 25.5, 23.7, 26.9; behind 64 others: 13 65, 62.5,
//     64.5; behind 1900: 7 37, 33, 23; 10 38, 33.2, 27.6; 13 39, 34, 33.  So from four parts on (three are worth it behind long windows alone).
//   24 and 32 units of four waves, with no others, would be quicker whole, 26.7 and 28.5, than halved, 30.0 and 32.6; behind others it was not timed.
constexpr int MOST_PARTS = 16, PLACES = 32;              // parts of a unit; of all of an XCD's
struct RowsPlan {
    int first, units, whole;                             // of an XCD: its first unit, all of them, those that are neither cut nor halved
    int parts;                                           // of each of the others; 0: halves
};
template <int NW> __device__ inline RowsPlan rows_plan(const WindowLayout& L, int total, int xcd)
{
    constexpr int SLOTS = 256 / NW;
    RowsPlan p;
    p.first = (int)((long long)xcd * total / NUM_XCD);
    p.units = (int)((long long)(xcd + 1) * total / NUM_XCD) - p.first;
    const int full = p.units / SLOTS * SLOTS, rem = p.units - full;
    p.whole = rem <= SLOTS / 2 ? full : p.units;
    p.parts = rem > 0 && rem <= SLOTS / 2 ? min(PLACES / rem, L.most_parts) : 0;
    if (p.parts < (NW == 8 ? 2 : 4)) p.parts = 0;        // fewer are hardly ever quicker than halves, which leave no records
    return p;
}
// a part's record: per thread 64 sums, in groups of four, then m, l
template <int NW> struct Record {
    static constexpr int THREADS = 64 * NW, FLOATS = THREADS * (64 + 2);
    static __device__ float* at(void* workspace, int xcd, int place) { return (float*)workspace + (size_t)(xcd * PLACES + place) * FLOATS; }
};
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
// The row tiles of 64 requests from `from` on, as the lanes see them
template <int NW> struct Lines {
    static constexpr int WIDE_ROWS = NW * WAVE_ROWS;
    const BatchView& b;
    int new_len, prefix_len, cu, incl;
    __device__ int look(const WindowLayout& L, int from) // returns their number
    {
        const int lane = threadIdx.x & 63, r = min(from + lane, b.num_reqs - 1);
        new_len = b.new_lens[r];
        prefix_len = b.prefix_lens[r];
        cu = b.cu_new_lens[r];
        incl = scan64(from + lane < b.num_reqs ? tiles_of(L, new_len) : 0);
        return __builtin_amdgcn_readlane(incl, 63);
    }
    // of one request
    __device__ int tiles_of(const WindowLayout& L, int length) const { return (clamp_new_len(b, length, true) * L.G + WIDE_ROWS - 1) / WIDE_ROWS; }
    __device__ int total(const WindowLayout& L)
    {
        if (b.num_reqs <= 64) return look(L, 0);
        int sum = 0;                                     // of this lane's requests: their lengths travel together
        for (int r = threadIdx.x & 63; r < b.num_reqs; r += 64) sum += tiles_of(L, b.new_lens[r]);
        return __builtin_amdgcn_readlane(scan64(sum), 63);
    }
    // the n-th row tile of all, n < total(); half 0 or 1: that half of its rows
    __device__ bool take(const WindowLayout& L, const WindowView& w, int n, int half, Tile& t)
    {
        int from = 0;
        if (b.num_reqs > 64) {
            // which 64 requests it is among, 256 at a time
            const int lane = threadIdx.x & 63;
            for (;; from += 256) {
                int count[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int r = from + 64 * k + lane;
                    count[k] = r < b.num_reqs ? tiles_of(L, b.new_lens[r]) : 0;
                }
                bool here = from + 256 >= b.num_reqs;
#pragma unroll
                for (int k = 3; k >= 0; --k) count[k] = __builtin_amdgcn_readlane(scan64(count[k]), 63);
                if (n < count[0] + count[1] + count[2] + count[3]) here = true;
                if (!here) {
                    n -= count[0] + count[1] + count[2] + count[3];
                    continue;
                }
                int at = 0;
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (at == k && n >= count[k]) {
                        n -= count[k];
                        ++at;
                    }
                from += 64 * at;
                break;
            }
            if (from >= b.num_reqs) return false;
            look(L, from);
        }
        const unsigned long long hit = __builtin_amdgcn_ballot_w64(incl > n);
        if (hit == 0) return false;
        const int at = __builtin_ctzll(hit);
        const int length = __builtin_amdgcn_readlane(new_len, at), tiles = tiles_of(L, length);
        const int tile = n - (__builtin_amdgcn_readlane(incl, at) - tiles);
        return make_tile(b, L, w, from + at, (long long)tile * WIDE_ROWS + max(half, 0) * (WIDE_ROWS / 2), half >= 0 ? WIDE_ROWS / 2 : WIDE_ROWS, length,
                         __builtin_amdgcn_readlane(prefix_len, at), __builtin_amdgcn_readlane(cu, at), t);
    }
};

// compile-time loop: f(integral_constant<int, I>) for I = BEGIN .. END-1
template <int BEGIN, int END, class F>
__device__ __forceinline__ void static_for(F&& f)
{
    if constexpr (BEGIN < END) {
        f(std::integral_constant<int, BEGIN>{});
        static_for<BEGIN + 1, END>(f);
    }
}
// Ties a value to the place where it is written: the optimiser would gather such work in one clump elsewhere.  Emits nothing.
__device__ __forceinline__ void pin(float& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void pin(uint32_t& x) { asm volatile("" : "+v"(x)); }

__device__ inline bool is_finite_bf16(uint32_t half) { return (half & 0x7f80u) != 0x7f80u; }

enum Shape { ROWS, HALVED /* rows, of half a unit */, KEYS };
template <int SHAPE, int NW> struct Sizes {
    static constexpr int TILE = SHAPE == KEYS ? 32 : 64;                     // keys of a tile
    static constexpr int TILE_BYTES = TILE * D * 2;                          // of K, or of V
    static constexpr int RING = 4 * TILE_BYTES;                              // two slots of K and V
    static constexpr int OUT = NW * WAVE_ROWS * OUT_STRIDE;          // rows shapes: what is staged at the end; a halved unit's sums are less
    static constexpr int LDS = SHAPE == KEYS ? NW * RING : RING > OUT ? RING : OUT;
};

// The rows of tile t by the workgroup, or, of `parts`, part `part` of their keys, whose record is number `place` (of those that the keys shape leaves,
// or of the XCD's).  bad_s: rows shapes, which waves have taken an infinity or NaN of V out.
template <int SHAPE, int NW>
__device__ __forceinline__ void attend_tile(const AttnArgs& a, const WindowView& w, const WindowLayout& L, const Tile& t, int kvh, int parts, int part, int place,
                                            unsigned char* smem, int* bad_s)
{
    constexpr bool KEYS = SHAPE == Shape::KEYS, HALVED = SHAPE == Shape::HALVED;
    constexpr int TB = Sizes<SHAPE, NW>::TILE / BLK, TILE_BYTES = Sizes<SHAPE, NW>::TILE_BYTES, RING = Sizes<SHAPE, NW>::RING;
    constexpr int KB = SHAPE == ROWS ? 2 : 1;            // 32-key parts of a tile that a wave takes
    // rows shapes: the waves of a block of the tile bring 4 INSTR rows of it each
    constexpr int PER_BLOCK = KEYS ? 1 : NW / TB, INSTR = 4 / PER_BLOCK;
    const BatchView& b = a.b;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, h32 = lane >> 5;
    const int G = L.G;

    // this workgroup's tiles, and of those this wave's
    const int all_tiles = (t.blocks + TB - 1) / TB;
    int t_begin = 0, t_end = all_tiles;
    if (KEYS || (SHAPE == ROWS && parts > 1)) {
        const int share = KEYS ? share_of(all_tiles, parts, L.by_parts, MIN_TILES_KEYS) : share_of(all_tiles, parts);
        t_begin = part * share;                              // (at most the tiles and a share for each part more)
        if (t_begin >= all_tiles) return;
        t_end = min(t_begin + share, all_tiles);
        if (share >= all_tiles) parts = 1;                   // this one does it all
    }
    const int step = KEYS ? NW : 1, t_first = KEYS ? t_begin + wave : t_begin;
    const int n_mine = t_end > t_first ? (t_end - t_first + step - 1) / step : 0;

    const int wrow0 = t.row0 + (KEYS ? 0 : HALVED ? wave >> 1 : wave) * WAVE_ROWS;
    const int kb0 = HALVED ? wave & 1 : 0;               // of a tile's 32-key parts the first that this wave takes
    const bool active = wrow0 < t.n_rows;                // (a wave without rows only fetches)
    const int row_c = min(wrow0 + l32, t.n_rows - 1);
    const int tok = L.by_G.quotient(row_c);
    const int limit = t.P + tok, low = window_low(w, limit);             // of this lane's row
    const int limit_min = t.P + L.by_G.quotient(min(wrow0, t.n_rows - 1));
    const int low_max = window_low(w, t.P + L.by_G.quotient(min(wrow0 + WAVE_ROWS, t.n_rows) - 1));

    const __bf16* __restrict__ qp = (const __bf16*)a.q + (((long long)t.first_row + tok) * b.num_q_heads + kvh * G + (row_c - tok * G)) * D + 8 * h32;
    bf16x8 qf[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *(const bf16x8*)(qp + 16 * s);

    // ---- fetching.  An instruction brings 4 rows of 256 bytes; lane i lands on row i / 16, chunk i % 16, and takes the chunk that belongs there.
    //        K: row = 16 block + swap23(key in block), chunk c of it at c ^ (row & 15)    (read with ds_read_b128)
    //        V: row = key,                             chunk c of it at c ^ ((row & 3) << 2)      (read with ds_read_tr16_b64)
    const int ld_row = lane >> 4, ld_p = lane & 15;
    const int my_block = KEYS ? 0 : wave / PER_BLOCK, j0 = KEYS ? 0 : wave % PER_BLOCK * INSTR;      // of a tile; its first 4 j0 rows are another wave's
    int k_goff[INSTR];
#pragma unroll
    for (int j = 0; j < INSTR; ++j) k_goff[j] = swap23(4 * (j0 + j) + ld_row) * 256 + ((ld_p ^ (4 * (j0 + j) + ld_row)) << 4);
    const int v_goff = (4 * j0 + ld_row) * 256 + ((ld_p ^ (ld_row << 2)) << 4);
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem + (KEYS ? wave * RING : 0);
    unsigned char* const my_ring = smem + (KEYS ? wave * RING : 0);
    const int32_t* __restrict__ pt = b.page_table + (long long)t.r * b.max_pages;
    const unsigned char* const kcb = (const unsigned char*)a.k_cache;
    const unsigned char* const vcb = (const unsigned char*)a.v_cache;
    // Where this wave's blocks lie, in slabs of the pool: lane k has that of the k-th block it fetches (KEYS: two of each of its tiles, else one of each
    // tile) from its tile id_base on.  Behind the list's end the last block again: its keys are hidden from all rows.
    constexpr int PER_TILE = KEYS ? TB : 1, IDS = 64 / PER_TILE;
    int id_base = 0;
    auto slab_of_block = [&](int blk) {
        const int page = min(max(pt[min(blk >> b.page_shift, b.max_pages - 1)], 0), b.num_pages - 1);
        return (long long)((((long long)page * b.num_kv_heads + kvh) << b.page_shift) + (blk & ((1 << b.page_shift) - 1)));
    };
    long long id_vec = 0;
    auto refill = [&](int i) {
        const int tile = t_first + (i + lane / PER_TILE) * step;
        const int v = min(tile * TB + (KEYS ? lane % PER_TILE : my_block), t.blocks - 1);
        id_vec = slab_of_block(t.block(v));
        id_base = i;
    };
    auto slab = [&](int i, int which) -> long long {         // byte offset of the block
        const int at = (i - id_base) * PER_TILE + which;
        const uint32_t lo = __builtin_amdgcn_readlane((int)id_vec, at), hi = __builtin_amdgcn_readlane((int)(id_vec >> 32), at);
        return (long long)(((unsigned long long)hi << 32) | lo) * SLAB;
    };
    // this wave's share of its tile i (KEYS: all of it), into slot i % 2
    auto fetch_k = [&](int i) {
#pragma unroll
        for (int which = 0; which < PER_TILE; ++which) {
            const unsigned char* from = kcb + slab(i, which);
            const uint32_t to = ring + (i & 1) * TILE_BYTES + (KEYS ? which : my_block) * SLAB + j0 * 1024;
#pragma unroll
            for (int j = 0; j < INSTR; ++j) lds_dma16(from, k_goff[j], to + j * 1024);
        }
    };
    auto fetch_v = [&](int i) {
#pragma unroll
        for (int which = 0; which < PER_TILE; ++which) {
            const unsigned char* from = vcb + slab(i, which);
            const uint32_t to = ring + (2 + (i & 1)) * TILE_BYTES + (KEYS ? which : my_block) * SLAB + j0 * 1024;
#pragma unroll
            for (int j = 0; j < INSTR; ++j) lds_dma16(from, v_goff + j * 1024, to + j * 1024);
        }
    };
    // is block v of the list seen whole by all rows of this wave?  (by all of a tile's blocks: no masks)
    const int clear_lo = t.sink_blocks + (max(low_max, t.low_first) + BLK - 1) / BLK - t.low_first / BLK;
    const int clear_hi = (limit_min + 1) / BLK - t.gap;
    const int clear_sinks = min(min((int)((uint32_t)w.sinks / BLK), t.sink_blocks), (limit_min + 1) / BLK);
    auto clear = [&](int tile) { return (tile * TB >= clear_lo && (tile + 1) * TB <= clear_hi) || (tile + 1) * TB <= clear_sinks; };
    // the same for all rows of the workgroup: does V need looking at?
    const int wg_lo = t.sink_blocks + (t.low_last + BLK - 1) / BLK - t.low_first / BLK;
    const int wg_hi = (t.P + L.by_G.quotient(t.row0) + 1) / BLK - t.gap;
    const int wg_sinks = min(clear_sinks, wg_hi + t.gap);
    auto wg_clear = [&](int tile) { return (tile * TB >= wg_lo && (tile + 1) * TB <= wg_hi) || (tile + 1) * TB <= wg_sinks; };

    // V rows of a block that this wave fetched: those that no row of the workgroup sees become zeros, and in the others what is not
    // finite.  Returns which rows held such values.
    auto look_at_v = [&](int v, unsigned char* block) -> int {
        const int key0 = t.block(v) * BLK;
        int bad = 0;
#pragma unroll 1
        for (int jj = 0; jj < INSTR; ++jj) {
            const int j = j0 + jj, key = key0 + 4 * j + ld_row;
            uint4* at = (uint4*)(block + j * 1024 + lane * 16);
            const bool hidden = key > t.last || (key < t.low_first && key >= w.sinks);
            uint4 x = *at;
            uint32_t d[4] = {x.x, x.y, x.z, x.w};
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool lo = is_finite_bf16(d[e]), hi = is_finite_bf16(d[e] >> 16);
                odd = odd || !lo || !hi;
                d[e] = hidden ? 0u : d[e] & ((lo ? 0xffffu : 0u) | (hi ? 0xffff0000u : 0u));
            }
            if (hidden || odd) *at = make_uint4(d[0], d[1], d[2], d[3]);
            const unsigned long long lanes = __builtin_amdgcn_ballot_w64(odd && !hidden);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if ((lanes >> (16 * k)) & 0xffffull) bad |= 1 << (4 * j + k);
        }
        return bad;
    };

    // ---- LDS read addresses
    const int k_rd = l32 * 256 + ((h32 ^ (l32 & 15)) << 4);                  // step st: ^ (st << 5)
    const int v_rd = 2 * TILE_BYTES + (8 * h32 + ((lane & 15) >> 2)) * 256 +
                     ((4 * ((lane & 15) >> 2) + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) << 4) + (lane & 1) * 8;       // channel block nb: ^ (nb << 6)

    const float c_log2 = b.softmax_scale * LOG2E;
    float m = -INFINITY, l = 0.f;                            // reference (times log2 e); sum of this lane's weights
    // Lane n: which rows of V that this wave brought of the n-th tile looked at held what is not finite, 16 bits a block.  Tiles looked at hold a slot that some
    // rows see and others do not.  A tile's rows are of at most as many tokens, so that such slots lie in ROWS / 16 + 1 blocks at either end of a window, and in one
    // at the sinks' end, and n blocks in a row touch (n + 2 TB - 2) / TB tiles at most: 12 of eight waves (11 are reached), 8 of four, 6 of the keys shape.
    constexpr int MOST_LOOKED = 2 * (((KEYS ? 1 : NW) * WAVE_ROWS / BLK + 2 + 2 * TB - 2) / TB);
    static_assert(MOST_LOOKED <= 64, "a lane for each tile that is looked at");
    int odd_rows = 0, looked = 0;
    f32x16 o[4];
#pragma unroll
    for (int nb = 0; nb < 4; ++nb)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[nb][v] = 0.f;

    // S^T = K Q^T of this wave's tile i
    auto multiply_k = [&](int i, f32x16 (&s)[KB]) {
        const unsigned char* k = my_ring + (i & 1) * TILE_BYTES + kb0 * 32 * 256;
#pragma unroll
        for (int st = 0; st < 8; ++st)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const bf16x8 kf = *(const bf16x8*)(k + kb * 32 * 256 + (k_rd ^ (st << 5)));
                if (st == 0) {
                    f32x16 zero;
#pragma unroll
                    for (int v = 0; v < 16; ++v) zero[v] = 0.f;
                    s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[st], zero, 0, 0, 0);
                } else {
                    s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[st], s[kb], 0, 0, 0);
                }
            }
    };
    auto mask = [&](int tile, f32x16 (&s)[KB]) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // bit e: is key key0 + e seen?  The first `upto` are not behind the row's own, the first `before` are before its window, `first` are sinks.
                const int key0 = t.block(tile * TB + 2 * (kb0 + kb) + h) * BLK + 8 * h32;
                auto bits = [](int n) { return (1u << min(max(n, 0), 8)) - 1u; };
                const uint32_t seen = bits(limit - key0 + 1) & (~bits(low - key0) | bits(w.sinks - key0));
#pragma unroll
                for (int e = 0; e < 8; ++e) s[kb][8 * h + e] = (seen & (1u << e)) != 0 ? s[kb][8 * h + e] : -INFINITY;
            }
    };
    auto top_of = [&](const f32x16 (&s)[KB]) {               // the largest of this lane's scores
        float top = s[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) top = fmaxf(top, s[kb][v]);
        return top * c_log2;
    };
    // scores whose largest in this lane is `top` are next: is the reference far enough up?
    auto raise = [&](float top) {
        if (__builtin_amdgcn_ballot_w64(top > m + LAG) != 0) {
            const float both = pair_max(top);                // (both halves of a row decide alike)
            const bool up = both > m + LAG;
            const float alpha = up ? __builtin_amdgcn_exp2f(m - both) : 1.f;
            m = up ? both : m;
            l *= alpha;
#pragma unroll
            for (int nb = 0; nb < 4; ++nb)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[nb][v] *= alpha;
        }
    };
    typedef uint32_t Weights[KB][2][4];
    auto weigh = [&](const f32x16 (&s)[KB], Weights& p) {
        const float ref = m == -INFINITY ? 0.f : m;          // a row that has seen no key yet: its weights are zeros
        float sum0 = 0.f, sum1 = 0.f;                        // of the weights as they are, before they are rounded for the product: lse has 32 bits
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; v += 2) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(s[kb][v], c_log2, -ref)), p1 = __builtin_amdgcn_exp2f(fmaf(s[kb][v + 1], c_log2, -ref));
                sum0 += p0;
                sum1 += p1;
                bf16x2 pr;
                pr[0] = (__bf16)p0;
                pr[1] = (__bf16)p1;
                p[kb][v >> 3][(v & 7) >> 1] = __builtin_bit_cast(uint32_t, pr);
            }
        l += sum0 + sum1;
    };
    // O^T += V^T P^T
    auto multiply_v = [&](int i, const Weights& p) {
        const unsigned char* tile = my_ring + (i & 1) * TILE_BYTES + kb0 * 32 * 256;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
                const u32x4 pw = {p[kb][h][0], p[kb][h][1], p[kb][h][2], p[kb][h][3]};
                const bf16x8 pf = __builtin_bit_cast(bf16x8, pw);
#pragma unroll
                for (int nb = 0; nb < 4; ++nb) {
                    typedef short s16x4 __attribute__((ext_vector_type(4)));
                    const unsigned char* src = tile + (32 * kb + 16 * h) * 256 + (v_rd ^ (nb << 6));
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src));
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src + 4 * 256));
                    const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    o[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[nb], 0, 0, 0);
                }
            }
    };
    // What is not finite, to the rows that see it: sums that it is in are infinite or NaN whatever its weight.  Rows `bad` of block v of the list.
    auto add_odd = [&](int v, int bad) {
        const int blk = t.block(v);
        const long long at = slab_of_block(blk) * SLAB;
        for (int rest = bad; rest != 0; rest &= rest - 1) {
            const int place = __builtin_ctz(rest), key = blk * BLK + place;
            const bool seen = key <= limit && (key >= low || key < w.sinks);
#pragma unroll
            for (int nb = 0; nb < 4; ++nb)
#pragma unroll
                for (int v4 = 0; v4 < 4; ++v4) {
                    const uint2 x = *(const uint2*)(vcb + at + place * 256 + 2 * (32 * nb + 8 * v4 + 4 * h32));
                    const uint32_t half[4] = {x.x & 0xffffu, x.x >> 16, x.y & 0xffffu, x.y >> 16};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (seen && !is_finite_bf16(half[e])) o[nb][4 * v4 + e] += __uint_as_float(half[e] << 16);
                }
        }
    };

    if (n_mine > 0) {
        // Tile i + 1's scores are made while tile i's become weights: K is a tile ahead of V.
        f32x16 s0[KB], s1[KB];
        float top = 0.f;
        refill(0);
        fetch_k(0);
        fetch_v(0);
        if (n_mine > 1) fetch_k(1);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if constexpr (!KEYS) __syncthreads();
        if (active) {
            multiply_k(0, s0);
            if (!clear(t_first)) mask(t_first, s0);
            top = top_of(s0);
        }
        // V(i) and K(i + 1) are there, the next ones are asked for
        auto arrive = [&](int i) {
            const int tile = t_first + i * step;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (!wg_clear(tile)) {
                int bad = 0;
#pragma unroll 1
                for (int which = 0; which < PER_TILE; ++which)
                    bad |= look_at_v(tile * TB + (KEYS ? which : my_block), my_ring + (2 + (i & 1)) * TILE_BYTES + (KEYS ? which : my_block) * SLAB) << (16 * which);
                odd_rows = lane == looked ? bad : odd_rows;
                ++looked;
            }
            if constexpr (KEYS) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // all reads of the other slots are done, and V's zeros are written
            } else {
                __syncthreads();                             // everyone's share; and everyone is past its reads of the other slots
            }
            if (i + 2 - id_base >= IDS) refill(i + 1);
            if (KEYS || !active) {
                if (i + 1 < n_mine) fetch_v(i + 1);
                if (i + 2 < n_mine) fetch_k(i + 2);
            }
        };
        // One MFMA a slice, fenced, so that the order is the one written here: the matrix pipe has an instruction in every slice, its operand
        // was read from LDS AHEAD slices before, and the softmax fills the slots between.
        //   8 KB slices   S^T(i + 1) = K Q^T
        //   8 KB slices   O^T += V^T P^T
        // Beside both tile i's weights, two pairs in three slices: scaled, exponentials, then sums and rounding; beside the last the largest of the new scores.
        // (With a pair a slice, done with the scores, those slices were bound by the softmax and the others by the products, and the waves of a SIMD are in step.)
        auto iteration = [&](int i, auto parity, f32x16 (&now)[KB], f32x16 (&next)[KB]) {
            constexpr int R = decltype(parity)::value, N = 8 * KB, AHEAD = 2;
            arrive(i);
            if (!active) return;
            const unsigned char* k_tile = my_ring + (R ^ 1) * TILE_BYTES + kb0 * 32 * 256;
            const unsigned char* v_tile = my_ring + R * TILE_BYTES + kb0 * 32 * 256;
            auto read = [&](auto n) -> bf16x8 {              // operand of slice n
                constexpr int k = decltype(n)::value;
                if constexpr (k < N) {
                    return *(const bf16x8*)(k_tile + (k % KB) * 32 * 256 + (k_rd ^ ((k / KB) << 5)));
                } else {
                    typedef short s16x4 __attribute__((ext_vector_type(4)));
                    constexpr int block = (k - N) / 4, nb = (k - N) % 4;
                    const unsigned char* src = v_tile + 16 * block * 256 + (v_rd ^ (nb << 6));
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src));
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src + 4 * 256));
                    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                }
            };
            bf16x8 operand[2 * N + AHEAD];
            static_for<0, AHEAD>([&](auto n) { operand[decltype(n)::value] = read(n); });
            raise(top);
            const float ref = m == -INFINITY ? 0.f : m;      // a row that has seen no key yet: its weights are zeros
            uint32_t p[KB][2][4];
            float x[2][N], sum0 = 0.f, sum1 = 0.f;           // sums of the weights as they are, before they are rounded for the product: lse has 32 bits
            auto scaled = [&](auto n) {
                constexpr int u = decltype(n)::value;
                x[0][u] = fmaf(now[u >> 3][2 * (u & 7)], c_log2, -ref);
                x[1][u] = fmaf(now[u >> 3][2 * (u & 7) + 1], c_log2, -ref);
                pin(x[0][u]);
                pin(x[1][u]);
            };
            auto raised = [&](auto n) {
                constexpr int u = decltype(n)::value;
                x[0][u] = __builtin_amdgcn_exp2f(x[0][u]);
                x[1][u] = __builtin_amdgcn_exp2f(x[1][u]);
                pin(x[0][u]);
                pin(x[1][u]);
            };
            auto rounded = [&](auto n) {
                constexpr int u = decltype(n)::value;
                sum0 += x[0][u];
                sum1 += x[1][u];
                bf16x2 pr;
                pr[0] = (__bf16)x[0][u];
                pr[1] = (__bf16)x[1][u];
                uint32_t& to = p[u >> 3][(u >> 2) & 1][u & 3];
                to = __builtin_bit_cast(uint32_t, pr);
                pin(to);
                pin(sum0);
                pin(sum1);
            };
            // a pair's three steps, a slice apart, begin at slice SPREAD / 10 times its number: before they are needed, and over as many slices as may be
            constexpr int SPREAD = KB == 2 ? 15 : 14;
            auto soften = [&](auto n) {
                constexpr int k = decltype(n)::value;
                static_for<0, N>([&](auto pair) {
                    constexpr int from = decltype(pair)::value * SPREAD / 10;
                    if constexpr (k == from + 1) raised(pair);
                });
                static_for<0, N>([&](auto pair) {
                    constexpr int from = decltype(pair)::value * SPREAD / 10;
                    if constexpr (k == from + 2) rounded(pair);
                });
                static_for<0, N>([&](auto pair) {
                    constexpr int from = decltype(pair)::value * SPREAD / 10;
                    if constexpr (k == from) scaled(pair);
                });
            };
            __builtin_amdgcn_sched_barrier(0);
            static_for<0, N>([&](auto n) {
                constexpr int k = decltype(n)::value, kb = k % KB, st = k / KB;
                operand[k + AHEAD] = read(std::integral_constant<int, k + AHEAD>{});
                if constexpr (st == 0) {
                    f32x16 zero;
#pragma unroll
                    for (int v = 0; v < 16; ++v) zero[v] = 0.f;
                    next[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand[k], qf[st], zero, 0, 0, 0);
                } else {
                    next[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand[k], qf[st], next[kb], 0, 0, 0);
                }
                // (rows shapes: in between, and past the last tile the list's last blocks again, which costs less than a branch)
                if constexpr (!KEYS && k == 1) fetch_v(i + 1);
                if constexpr (!KEYS && k == 3) fetch_k(i + 2);
                soften(n);
                __builtin_amdgcn_sched_barrier(0);
            });
            auto product = [&](auto n) {
                constexpr int k = decltype(n)::value, block = k / 4, nb = k % 4;
                if constexpr (N + k + AHEAD < 2 * N) operand[N + k + AHEAD] = read(std::integral_constant<int, N + k + AHEAD>{});
                typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
                const u32x4 pw = {p[block >> 1][block & 1][0], p[block >> 1][block & 1][1], p[block >> 1][block & 1][2], p[block >> 1][block & 1][3]};
                o[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand[N + k], __builtin_bit_cast(bf16x8, pw), o[nb], 0, 0, 0);
                soften(std::integral_constant<int, N + k>{});
            };
            constexpr int FIRST = N / 2;                     // value products before the new scores are looked at
            static_for<0, FIRST>([&](auto n) {
                product(n);
                __builtin_amdgcn_sched_barrier(0);
            });
            if (!clear(t_first + (i + 1) * step)) {
                mask(t_first + (i + 1) * step, next);
                __builtin_amdgcn_sched_barrier(0);
            }
            float most = -INFINITY;
            static_for<FIRST, N>([&](auto n) {
                constexpr int k = decltype(n)::value, VALUES = 16 * KB, lo = (k - FIRST) * VALUES / (N - FIRST), hi = (k + 1 - FIRST) * VALUES / (N - FIRST);
                product(n);
                static_for<lo, hi>([&](auto v) { most = fmaxf(most, next[decltype(v)::value >> 4][decltype(v)::value & 15]); });
                pin(most);
                __builtin_amdgcn_sched_barrier(0);
            });
            l += sum0 + sum1;
            top = most * c_log2;
        };
        using even = std::integral_constant<int, 0>;
        using odd = std::integral_constant<int, 1>;
        int i = 0;
        for (; i + 2 < n_mine; i += 2) {
            iteration(i, even{}, s0, s1);
            iteration(i + 1, odd{}, s1, s0);
        }
        if (i + 1 < n_mine) {
            iteration(i, even{}, s0, s1);
            ++i;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) s0[kb] = s1[kb];
        }
        arrive(i);
        if (active) {
            Weights p;
            raise(top);
            weigh(s0, p);
            multiply_v(i, p);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // (what was fetched past the last tile)
    // what was not finite and taken out, to the rows that see it
    bool any = __builtin_amdgcn_ballot_w64(odd_rows != 0) != 0;
    if constexpr (!KEYS) {
        if (lane == 0) bad_s[wave] = any ? 1 : 0;
        __syncthreads();                                     // (and the rings are free)
        any = false;
#pragma unroll
        for (int k = 0; k < NW; ++k) any = any || __builtin_amdgcn_readfirstlane(bad_s[k]) != 0;
    }
    if (any) {
        int* list = (int*)my_ring;                           // [waves that brought blocks][64]
        if constexpr (!KEYS) {
            list[wave * 64 + lane] = odd_rows;
            __syncthreads();
        }
        int n = 0;
        for (int i = 0; i < n_mine; ++i) {
            const int tile = t_first + i * step;
            if (wg_clear(tile)) continue;
            for (int k = KEYS ? 0 : 2 * kb0; k < (HALVED ? 2 * kb0 + 2 : TB); ++k) {
                int rows = 0;
                if constexpr (KEYS) {
                    rows = __builtin_amdgcn_readlane(odd_rows, n) >> (16 * k) & 0xffff;
                } else {
                    for (int x = 0; x < PER_BLOCK; ++x) rows |= __builtin_amdgcn_readfirstlane(list[(k * PER_BLOCK + x) * 64 + n]);
                }
                if (rows != 0 && active) add_odd(tile * TB + k, rows);
            }
            ++n;
        }
    }
    const float l_row = pair_sum(l);
    auto at_row = [&](int row) -> long long {                // row of [T][H]
        const int token = L.by_G.quotient(row);
        return ((long long)t.first_row + token) * b.num_q_heads + kvh * G + (row - token * G);
    };
    __syncthreads();                                         // the rings are free

    if constexpr (!KEYS) {
        // out through LDS, so that an instruction stores four whole rows
        float l_all = l_row;
        if constexpr (HALVED) {
            // the second wave's sums to the first, lane by lane
            float* theirs = (float*)smem + (wave >> 1) * 64 * 66;
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            if (kb0 == 1) {
#pragma unroll
                for (int nb = 0; nb < 4; ++nb)
#pragma unroll
                    for (int v4 = 0; v4 < 4; ++v4)
                        *(f32x4*)(theirs + ((4 * nb + v4) * 64 + lane) * 4) = f32x4{o[nb][4 * v4], o[nb][4 * v4 + 1], o[nb][4 * v4 + 2], o[nb][4 * v4 + 3]};
                *(f32x2*)(theirs + 64 * 64 + 2 * lane) = f32x2{m, l_row};
            }
            __syncthreads();
            if (kb0 == 0) {
                const f32x2 ml = *(const f32x2*)(theirs + 64 * 64 + 2 * lane);
                const float top = fmaxf(m, ml[0]);
                const float mine = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top), other = ml[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0] - top);
                m = top;
                l_all = l_row * mine + ml[1] * other;
#pragma unroll
                for (int nb = 0; nb < 4; ++nb)
#pragma unroll
                    for (int v4 = 0; v4 < 4; ++v4) {
                        const f32x4 x = *(const f32x4*)(theirs + ((4 * nb + v4) * 64 + lane) * 4);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[nb][4 * v4 + e] = o[nb][4 * v4 + e] * mine + x[e] * other;
                    }
            }
            __syncthreads();                                 // what is staged next lies there
        }
        if (!active || kb0 != 0) return;
        if (SHAPE == ROWS && parts > 1) {
            float* rec = Record<NW>::at(a.workspace, blockIdx.x % NUM_XCD, place);
#pragma unroll
            for (int nb = 0; nb < 4; ++nb)
#pragma unroll
                for (int v4 = 0; v4 < 4; ++v4)
                    *(f32x4*)(rec + ((4 * nb + v4) * Record<NW>::THREADS + tid) * 4) = f32x4{o[nb][4 * v4], o[nb][4 * v4 + 1], o[nb][4 * v4 + 2], o[nb][4 * v4 + 3]};
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            *(f32x2*)(rec + 64 * Record<NW>::THREADS + 2 * tid) = f32x2{m, l_all};
            return;
        }
        const float inv = l_all != 0.f ? 1.f / l_all : 0.f;  // (a row sees itself)
        unsigned char* stage = smem + wave * (32 * OUT_STRIDE);
#pragma unroll
        for (int nb = 0; nb < 4; ++nb)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4) {
                bf16x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (__bf16)(o[nb][4 * v4 + e] * inv);
                *(bf16x4*)(stage + l32 * OUT_STRIDE + 2 * (32 * nb + 8 * v4 + 4 * h32)) = x;
            }
        if (a.lse != nullptr && h32 == 0 && wrow0 + l32 < t.n_rows) a.lse[at_row(wrow0 + l32)] = m * LN2 + logf(l_all);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = wrow0 + 4 * j + ld_row;
            if (row < t.n_rows)
                *(uint4*)((__bf16*)a.out + at_row(row) * D + ld_p * 8) = *(const uint4*)(stage + (4 * j + ld_row) * OUT_STRIDE + ld_p * 16);
        }
    } else {
        // the waves' sums: rows of REC_STRIDE floats
        float* mine = (float*)smem + wave * WAVE_ROWS * REC_STRIDE + l32 * REC_STRIDE;
#pragma unroll
        for (int nb = 0; nb < 4; ++nb)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4)
                *(f32x4*)(mine + 32 * nb + 8 * v4 + 4 * h32) = f32x4{o[nb][4 * v4], o[nb][4 * v4 + 1], o[nb][4 * v4 + 2], o[nb][4 * v4 + 3]};
        if (h32 == 0) {
            mine[D] = m;
            mine[D + 1] = l_row;
        }
        __syncthreads();
        // 8 threads a row, 16 channels each
        const int row = tid >> 3, ch = (tid & 7) * 4;
        if (t.row0 + row >= t.n_rows) return;
        const float* first = (const float*)smem + row * REC_STRIDE;
        float top = -INFINITY, total = 0.f, weight[WAVES];
#pragma unroll
        for (int k = 0; k < WAVES; ++k) top = fmaxf(top, first[k * WAVE_ROWS * REC_STRIDE + D]);
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
            const float mk = first[k * WAVE_ROWS * REC_STRIDE + D];
            weight[k] = mk == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mk - top);
            total += weight[k] * first[k * WAVE_ROWS * REC_STRIDE + D + 1];
        }
        f32x4 sum[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            sum[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < WAVES; ++k) sum[x] += weight[k] * *(const f32x4*)(first + k * WAVE_ROWS * REC_STRIDE + ch + 32 * x);
        }
        if (parts > 1) {
            float* rec = (float*)a.workspace + ((long long)place * WAVE_ROWS + row) * REC_STRIDE;
#pragma unroll
            for (int x = 0; x < 4; ++x) *(f32x4*)(rec + ch + 32 * x) = sum[x];
            if (ch == 0) {
                rec[D] = top;
                rec[D + 1] = total;
            }
            return;
        }
        const float inv = total != 0.f ? 1.f / total : 0.f;
        const long long at = at_row(t.row0 + row);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            bf16x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (__bf16)(sum[x][e] * inv);
            *(bf16x4*)((__bf16*)a.out + at * D + ch + 32 * x) = y;
        }
        if (a.lse != nullptr && ch == 0) a.lse[at] = top * LN2 + logf(total);
    }
}

__global__ __launch_bounds__(64 * WAVES, 1) void attn_window_keys_kernel(AttnArgs a, WindowView w, WindowLayout L)
{
    __shared__ __attribute__((aligned(1024))) unsigned char smem[Sizes<KEYS, WAVES>::LDS];
    const BatchView& b = a.b;
    int item = blockIdx.x, slot, part, kvh;
    if (L.per_xcd > 0) item = (blockIdx.x % NUM_XCD) * L.per_xcd + blockIdx.x / NUM_XCD;
    if (item >= L.items) return;
    if (L.per_xcd > 0) {                                 // neighbours share a KV head, and mostly a request
        const int group = L.by_slots.quotient(item);
        slot = item - group * L.slots;
        kvh = L.by_parts.quotient(group);
        part = group - kvh * L.parts;
    } else {
        const int pair = L.by_parts.quotient(item);
        part = item - pair * L.parts;
        slot = L.by_kv_heads.quotient(pair);
        kvh = pair - slot * b.num_kv_heads;
    }
    Tile t;
    if (find_tile<WAVE_ROWS>(b, L, w, slot, t))
        attend_tile<KEYS, WAVES>(a, w, L, t, kvh, L.parts, part, (slot * b.num_kv_heads + kvh) * L.parts + part, smem, nullptr);
}

// ---- Decode shape: a request's one new token, at most 16 query heads on a KV head.  As the keys shape, with 16 rows in place of 32
// (v_mfma_f32_16x16x32_bf16: half of the products and exponentials) and without what only rows of several tokens need: all rows see the same keys.
// Scores: lane (query lane % 16, g = lane / 16) has keys 4 g .. 4 g + 3 of a block.  Two blocks' are its 8 of the value product's 32 keys, whatever order
// these have; V's operand is read to match.
constexpr int DECODE_ROWS = 16;
__device__ inline float quad_max(float x)                    // over the four lanes of a query
{
    const uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ inline float quad_sum(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
template <bool STREAM>
__global__ __launch_bounds__(64 * WAVES, 1) void attn_window_decode_kernel(AttnArgs a, WindowView w, WindowLayout L)
{
    constexpr int TB = 2, TILE_BYTES = TB * SLAB, RING = 4 * TILE_BYTES;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[WAVES * RING];
    const BatchView& b = a.b;
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int pair = L.by_parts.quotient(blockIdx.x), part = blockIdx.x - pair * L.parts;
    const int slot = L.by_kv_heads.quotient(pair), kvh = pair - slot * b.num_kv_heads, G = L.G;
    const int new_len = b.new_lens[slot], prefix_len = b.prefix_lens[slot], cu = b.cu_new_lens[slot];
    // every argument that is needed further down travels with the lengths
    asm volatile("" ::"s"(a.q), "s"(a.k_cache), "s"(a.v_cache), "s"(a.out), "s"(a.lse), "s"(a.workspace), "s"(b.page_table), "s"(new_len), "s"(prefix_len), "s"(cu));
    Tile t;
    if (!make_tile(b, L, w, slot, 0, DECODE_ROWS, min(new_len, 1), prefix_len, cu, t)) return;
    const int32_t* __restrict__ pt = b.page_table + (long long)slot * b.max_pages;

    const int all_tiles = (t.blocks + TB - 1) / TB, share = share_of(all_tiles, L.parts, L.by_parts, MIN_TILES);
    const int t_begin = part * share, t_end = min(t_begin + share, all_tiles), t_first = t_begin + wave;
    if (t_begin >= all_tiles) return;
    const int n_mine = t_end > t_first ? (t_end - t_first + WAVES - 1) / WAVES : 0;

    // where this wave's blocks lie, in slabs of the pool: lane k has that of the k-th it fetches from its tile id_base on
    constexpr int IDS = 64 / TB;
    int id_base = 0;
    long long id_vec = 0;
    auto refill = [&](int i) {
        const int blk = t.block(min((t_first + (i + lane / TB) * WAVES) * TB + lane % TB, t.blocks - 1));
        const int page = min(max(pt[min(blk >> b.page_shift, b.max_pages - 1)], 0), b.num_pages - 1);
        id_vec = (((long long)page * b.num_kv_heads + kvh) << b.page_shift) + (blk & ((1 << b.page_shift) - 1));
        id_base = i;
    };
    if (n_mine > 0) refill(0);

    const __bf16* __restrict__ qp = (const __bf16*)a.q + ((long long)t.first_row * b.num_q_heads + kvh * G + min(l16, G - 1)) * D + 8 * g;
    bf16x8 qf[4];
#pragma unroll
    for (int st = 0; st < 4; ++st) qf[st] = *(const bf16x8*)(qp + 32 * st);

    // an instruction brings 4 rows of 256 bytes; chunk c of K's row lies at c ^ row, of V's at c ^ ((row & 3) << 2)
    const int ld_row = lane >> 4, ld_p = lane & 15;
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem + wave * RING;
    unsigned char* const my_ring = smem + wave * RING;
    const int k_goff = ld_row * 256 + ((ld_p ^ ld_row) << 4), v_goff = ld_row * 256 + ((ld_p ^ (ld_row << 2)) << 4);
    const unsigned char* const kcb = (const unsigned char*)a.k_cache;
    const unsigned char* const vcb = (const unsigned char*)a.v_cache;
    auto bring = [](const unsigned char* from, int offset, uint32_t to) {
        if constexpr (STREAM) lds_dma16_streamed(from, offset, to);
        else lds_dma16(from, offset, to);
    };
    auto fetch = [&](int i) {                                // tile i into slot i % 2
#pragma unroll
        for (int which = 0; which < TB; ++which) {
            const int at = (i - id_base) * TB + which;
            const uint32_t lo = __builtin_amdgcn_readlane((int)id_vec, at), hi = __builtin_amdgcn_readlane((int)(id_vec >> 32), at);
            const long long slab = (long long)(((unsigned long long)hi << 32) | lo) * SLAB;
            const uint32_t to = ring + (i & 1) * TILE_BYTES + which * SLAB;
#pragma unroll
            for (int j = 0; j < 4; ++j) bring(kcb + slab, (k_goff ^ (j << 6)) + j * 1024, to + j * 1024);
#pragma unroll
            for (int j = 0; j < 4; ++j) bring(vcb + slab, v_goff + j * 1024, to + 2 * TILE_BYTES + j * 1024);
        }
    };
    const int k_rd = l16 * 256 + ((g ^ l16) << 4);           // step st: ^ (st << 6)
    const int v_rd = 2 * TILE_BYTES + (4 * g + (l16 >> 2)) * 256 + ((4 * (l16 >> 2) + ((l16 & 3) >> 1)) << 4) + (l16 & 1) * 8;    // channel block nb: ^ (nb << 5)
    const int limit = t.last, low = t.low_first;
    auto seen = [&](int key) { return key <= limit && (key >= low || key < w.sinks); };
    auto seen_whole = [&](int key) { return key + BLK - 1 <= limit && (key >= low || key + BLK - 1 < w.sinks); };    // a block
    const float c_log2 = b.softmax_scale * LOG2E;
    float m = -INFINITY, l = 0.f;
    f32x4 o[8];
#pragma unroll
    for (int nb = 0; nb < 8; ++nb) o[nb] = f32x4{0.f, 0.f, 0.f, 0.f};

    if (n_mine > 0) {
        // (q is here before the first tile is asked for: the waits below count a tile's loads)
        asm volatile("" ::"v"(qf[0]), "v"(qf[1]), "v"(qf[2]), "v"(qf[3]) : "memory");
        fetch(0);
        for (int i = 0; i < n_mine; ++i) {
            const int tile = t_first + i * WAVES;
            // (reads of the other slot are done: their values have been used)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (i + 1 < n_mine) {
                if (i + 1 - id_base >= IDS) refill(i + 1);
                fetch(i + 1);
                asm volatile("s_waitcnt vmcnt(16)" ::: "memory");            // tile i's 16 loads are those before
            } else {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
            const int key0 = t.block(tile * TB) * BLK, key1 = t.block(tile * TB + 1) * BLK;
            const bool whole = seen_whole(key0) && seen_whole(key1);
            const unsigned char* at = my_ring + (i & 1) * TILE_BYTES;
            if (!whole) {
                // V of slots that are not seen: whatever they hold, times a weight of 0, must be 0
#pragma unroll
                for (int j = 0; j < 4 * TB; ++j) {
                    const int key = (j < 4 ? key0 : key1) + 4 * (j & 3) + ld_row;
                    if (!seen(key)) *(uint4*)(my_ring + (2 + (i & 1)) * TILE_BYTES + j * 1024 + lane * 16) = make_uint4(0, 0, 0, 0);
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
            f32x4 s[TB];
#pragma unroll
            for (int st = 0; st < 4; ++st)
#pragma unroll
                for (int u = 0; u < TB; ++u) {
                    const bf16x8 kf = *(const bf16x8*)(at + u * SLAB + (k_rd ^ (st << 6)));
                    s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[st], st == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[u], 0, 0, 0);
                }
            if (!whole)
#pragma unroll
                for (int u = 0; u < TB; ++u)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        if (!seen((u == 0 ? key0 : key1) + 4 * g + v)) s[u][v] = -INFINITY;
            float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))) * c_log2;
            if (__builtin_amdgcn_ballot_w64(top > m + LAG) != 0) {
                top = quad_max(top);                         // (all four lanes decide alike)
                const bool up = top > m + LAG;
                const float alpha = up ? __builtin_amdgcn_exp2f(m - top) : 1.f;
                m = up ? top : m;
                l *= alpha;
#pragma unroll
                for (int nb = 0; nb < 8; ++nb) o[nb] *= alpha;
            }
            const float ref = m == -INFINITY ? 0.f : m;
            bf16x8 pf;
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][e & 3], c_log2, -ref));
                sum += p;                                    // (as it is, before it is rounded for the product)
                pf[e] = (__bf16)p;
            }
            l += sum;
#pragma unroll
            for (int nb = 0; nb < 8; ++nb) {
                typedef short s16x4 __attribute__((ext_vector_type(4)));
                const unsigned char* src = at + (v_rd ^ (nb << 5));
                const s16x4 first = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src));
                const s16x4 second = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src + SLAB));
                const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(first, second, 0, 1, 2, 3, 4, 5, 6, 7));
                o[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, o[nb], 0, 0, 0);
            }
        }
    }
    // ---- the waves' sums: rows of REC_STRIDE floats
    l = quad_sum(l);
    __syncthreads();                                         // the rings are free
    float* mine = (float*)smem + (wave * DECODE_ROWS + l16) * REC_STRIDE;
#pragma unroll
    for (int nb = 0; nb < 8; ++nb) *(f32x4*)(mine + 16 * nb + 4 * g) = o[nb];
    if (g == 0) {
        mine[D] = m;
        mine[D + 1] = l;
    }
    __syncthreads();
    const int row = tid >> 4, ch = (tid & 15) * 4;           // 16 threads a row, 8 channels each
    if (row >= G) return;
    const float* first = (const float*)smem + row * REC_STRIDE;
    float top = -INFINITY, total = 0.f, weight[WAVES];
#pragma unroll
    for (int k = 0; k < WAVES; ++k) top = fmaxf(top, first[k * DECODE_ROWS * REC_STRIDE + D]);
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
        const float mk = first[k * DECODE_ROWS * REC_STRIDE + D];
        weight[k] = mk == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mk - top);
        total += weight[k] * first[k * DECODE_ROWS * REC_STRIDE + D + 1];
    }
    f32x4 sum[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        sum[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < WAVES; ++k) sum[x] += weight[k] * *(const f32x4*)(first + k * DECODE_ROWS * REC_STRIDE + ch + 64 * x);
    }
    if (share < all_tiles) {                                 // one of several parts
        float* rec = (float*)a.workspace + ((long long)(pair * L.parts + part) * DECODE_ROWS + row) * REC_STRIDE;
#pragma unroll
        for (int x = 0; x < 2; ++x) *(f32x4*)(rec + ch + 64 * x) = sum[x];
        if (ch == 0) {
            rec[D] = top;
            rec[D + 1] = total;
        }
        return;
    }
    const float inv = total != 0.f ? 1.f / total : 0.f;
    const long long at = (long long)t.first_row * b.num_q_heads + kvh * G + row;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (__bf16)(sum[x][e] * inv);
        *(bf16x4*)((__bf16*)a.out + at * D + ch + 64 * x) = y;
    }
    if (a.lse != nullptr && ch == 0) a.lse[at] = top * LN2 + logf(total);
}

template <int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_window_rows_kernel(AttnArgs a, WindowView w, WindowLayout L)
{
    __shared__ __attribute__((aligned(1024))) unsigned char smem[Sizes<ROWS, NW>::LDS];
    __shared__ int bad_s[NW];
    const BatchView& b = a.b;
    Lines<NW> lines = {b};
    const int tiles = lines.total(L), i = blockIdx.x / NUM_XCD;
    const RowsPlan plan = rows_plan<NW>(L, tiles * b.num_kv_heads, blockIdx.x % NUM_XCD);
    const bool whole = i < plan.whole;
    const int share = whole || plan.parts == 0 ? 2 : plan.parts, place = i - plan.whole;             // workgroups of a unit
    const int nth = whole ? i : plan.whole + place / share, part = whole ? 0 : place % share;
    if (nth >= plan.units) return;
    const int unit = plan.first + nth, kvh = unit / tiles;
    const bool halved = !whole && plan.parts == 0;
    Tile t;
    if (!lines.take(L, w, unit - kvh * tiles, halved ? part : -1, t)) return;
    if (halved) attend_tile<HALVED, NW>(a, w, L, t, kvh, 1, 0, 0, smem, bad_s);
    else attend_tile<ROWS, NW>(a, w, L, t, kvh, whole ? 1 : plan.parts, part, place, smem, bad_s);
}

// over all lanes of a wave
__device__ inline float wave_max(float x)
{
    for (int n = 1; n < 64; n *= 2) x = fmaxf(x, __shfl_xor(x, n));
    return x;
}
__device__ inline float wave_sum(float x)
{
    for (int n = 1; n < 64; n *= 2) x += __shfl_xor(x, n);
    return x;
}

// Adds the records of a row tile's parts up: a wave for a row, two channels a lane, AT_ONCE parts' rows on their way at a time.
// A record counts if there is that part, whatever its weight: 0 times a sum that an infinity or NaN is in is NaN, as in the waves' own sums.
constexpr int AT_ONCE = 16;
template <int ROWS>                                      // of a record
__global__ __launch_bounds__(64 * WAVES) void attn_window_merge_kernel(AttnArgs a, WindowView w, WindowLayout L, int row_groups)
{
    const BatchView& b = a.b;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int unit = blockIdx.x / row_groups, row = (blockIdx.x - unit * row_groups) * WAVES + wave;
    const int slot = L.by_kv_heads.quotient(unit), kvh = unit - slot * b.num_kv_heads;
    const float* rec = (const float*)a.workspace + ((long long)unit * L.parts * ROWS + min(row, ROWS - 1)) * REC_STRIDE;
    constexpr int STRIDE = ROWS * REC_STRIDE;
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    // Records travel with the lengths that say which of them there are: what the others hold is not looked at.
    f32x2 ml, v[AT_ONCE];
    auto ask_sums = [&](int k0) { ml = *(const f32x2*)(rec + (long long)min(k0 + lane, L.parts - 1) * STRIDE + D); };      // lane k: reference and sum of part k0 + k
    auto ask = [&](int k) {
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) v[u] = *(const f32x2*)(rec + (long long)min(k + u, L.parts - 1) * STRIDE + 2 * lane);
    };
    ask_sums(0);
    ask(0);
    Tile t;
    if (!find_tile<ROWS>(b, L, w, slot, t)) return;
    if (row >= ROWS || t.row0 + row >= t.n_rows) return;
    const int tiles = (t.blocks + 1) / 2, share = share_of(tiles, L.parts, L.by_parts, ROWS == DECODE_ROWS ? MIN_TILES : MIN_TILES_KEYS);       // (of 32 keys)
    if (share >= tiles) return;                              // in one part: done
    float top = -INFINITY, total = 0.f, x = 0.f, y = 0.f;
    for (int k0 = 0; k0 * share < tiles; k0 += 64) {
        if (k0 > 0) {
            ask_sums(k0);
            ask(k0);
        }
        const bool mine = (k0 + lane) * share < tiles;       // is there that part?
        const float m = mine ? ml[0] : -INFINITY;
        const float most = fmaxf(top, wave_max(m));
        const float before = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - most), weight = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - most);
        top = most;
        total = total * before + wave_sum(mine ? weight * ml[1] : 0.f);
        x *= before;
        y *= before;
        for (int k = k0; k < k0 + 64 && k * share < tiles; k += AT_ONCE) {
            if (k > k0) ask(k);
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const float w_u = __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(weight), (k + u - k0) & 63));
                const bool there = (k + u) * share < tiles;
                x = there ? fmaf(w_u, v[u][0], x) : x;
                y = there ? fmaf(w_u, v[u][1], y) : y;
            }
        }
    }
    const float inv = total != 0.f ? 1.f / total : 0.f;
    const int token = L.by_G.quotient(t.row0 + row);
    const long long at = ((long long)t.first_row + token) * b.num_q_heads + kvh * L.G + (t.row0 + row - token * L.G);
    bf16x2 out;
    out[0] = (__bf16)(x * inv);
    out[1] = (__bf16)(y * inv);
    *(bf16x2*)((__bf16*)a.out + at * D + 2 * lane) = out;
    if (a.lse != nullptr && lane == 0) a.lse[at] = top * LN2 + logf(total);
}

// The same for the rows shape's cut units.  SUB workgroups for each of a unit's parts share its sums: 16 groups of four of each of its threads.
constexpr int SUB = 4;
template <int NW>
__global__ __launch_bounds__(256) void attn_window_rows_merge_kernel(AttnArgs a, WindowView w, WindowLayout L)
{
    constexpr int THREADS = Record<NW>::THREADS;
    const BatchView& b = a.b;
    const int xcd = blockIdx.x % NUM_XCD, at_place = blockIdx.x / NUM_XCD / SUB, sub = blockIdx.x / NUM_XCD % SUB;
    Lines<NW> lines = {b};
    const int tiles = lines.total(L);
    const RowsPlan plan = rows_plan<NW>(L, tiles * b.num_kv_heads, xcd);
    if (plan.parts == 0 || at_place >= (plan.units - plan.whole) * plan.parts) return;
    const int nth = at_place / plan.parts, share = at_place - nth * plan.parts;
    const int unit = plan.first + plan.whole + nth, kvh = unit / tiles;
    Tile t;
    if (!lines.take(L, w, unit - kvh * tiles, -1, t)) return;
    const int tiles_here = (t.blocks + 3) / 4, share_here = share_of(tiles_here, plan.parts);        // (of 64 keys)
    if (share_here >= tiles_here) return;                    // in one part: done
    const int parts = (tiles_here + share_here - 1) / share_here;
    const float* rec = Record<NW>::at(a.workspace, xcd, nth * plan.parts);
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    for (int item = (share * SUB + sub) * 256 + threadIdx.x; item < 16 * THREADS; item += plan.parts * SUB * 256) {
        const int group = item / THREADS, col = item % THREADS, row = (col >> 6) * WAVE_ROWS + (col & 31), h32 = (col >> 5) & 1;
        if (t.row0 + row >= t.n_rows) continue;
        f32x4 v[MOST_PARTS];
        f32x2 ml[MOST_PARTS];
#pragma unroll
        for (int k = 0; k < MOST_PARTS; ++k)
            if (k < parts) {
                ml[k] = *(const f32x2*)(rec + (size_t)k * Record<NW>::FLOATS + 64 * THREADS + 2 * col);
                v[k] = *(const f32x4*)(rec + (size_t)k * Record<NW>::FLOATS + item * 4);
            }
        float top = -INFINITY, total = 0.f;
#pragma unroll
        for (int k = 0; k < MOST_PARTS; ++k)
            if (k < parts) top = fmaxf(top, ml[k][0]);
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < MOST_PARTS; ++k)
            if (k < parts) {
                const float weight = ml[k][0] != -INFINITY ? __builtin_amdgcn_exp2f(ml[k][0] - top) : 0.f;
                total += weight * ml[k][1];
                sum += weight * v[k];
            }
        const float inv = total != 0.f ? 1.f / total : 0.f;
        const int token = L.by_G.quotient(t.row0 + row);
        const long long at = ((long long)t.first_row + token) * b.num_q_heads + kvh * L.G + (t.row0 + row - token * L.G);
        bf16x4 out;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = (__bf16)(sum[e] * inv);
        *(bf16x4*)((__bf16*)a.out + at * D + 32 * (group >> 2) + 8 * (group & 3) + 4 * h32) = out;
        if (a.lse != nullptr && group == 0 && h32 == 0) a.lse[at] = top * LN2 + logf(total);
    }
}

constexpr int COMPUTE_UNITS = 256;
// K and V of a decode step, each read once, past the caches where they are more than the last-level cache keeps for a next call (537 MB 101 us through the caches
// and 90 past them, 800 ragged 308 and 276, 393 on 8 heads 81 and 70; 134 MB 29.0 and 29.3, 66 30.6 and 30.6).
constexpr long long STREAM_BYTES = 96ll << 20;
// The rows shape from so many units on (of 128 rows, one for each request at least), us in the rows and in the keys shape: 8 units, 36 tokens behind 2048 20.5 and
// 14.1; 12, 50 behind 1024 16.1 and 15.2; 16, 60 behind 4096 22.2 and 21.5, 4 x 9 behind 1024 14.3 and 18.0, behind 4096 18.5 and 26.5; 24, 100 behind
// 4096 25.4 and 31.6; 28, 160 behind 1024 17.9 and 22.7; 64, 16 x 9 behind 1024 19.4 and 32.1.
constexpr int ROWS_UNITS = 16;
// Tiles of 64 keys from which on a window is long: see RowsPlan.  us with four and with eight waves, each with its way to cut: 8 x 400 tokens behind 1024 (17 tiles) 78
// and 86, 1500 (24) 104 and 102, 2048 (33) 126 and 122, 4096 (65) 218 and 208; 2 x 2048 82 and 83, 112 and 108, 139 and 135, 255 and 245; 2 x 585 behind 1500 42 and
// 47, 2048 51 and 53, 4096 90 and 83; one of 250 21.8 and 24.8, 24.1 and 25.6, 33.7 and 33.3.
constexpr int LONG_TILES = 32;
constexpr int CUT_ROUNDS = 4;                            // a long window's last units are cut in batches of up to so many rounds, a short one's where they are all there is:
                                                         // beyond, what the second kernel takes (5 us where nothing was cut after all) is as much as there is to gain

// A request that may have no token has room for a row tile all the same: so many items at most are cut (no batch of 15 requests or fewer has more), or
// a few tokens among thousands of requests would want a workspace of gigabytes.
constexpr long long MOST_ITEMS = 4096;

// How a batch is dealt, from what the host knows.
struct Deal {
    int rows_waves;                                      // of a workgroup of the rows shape, 0: the others
    bool decode, stream;                                 // decode shape; its K and V past the caches
    WindowLayout L;
    long long grid;
    size_t workspace;
};
Deal deal_of(const BatchView& b, const WindowView& w)
{
    Deal s = {};
    const int G = b.num_q_heads / b.num_kv_heads;
    const long long rows = (long long)b.total_new_tokens * G;
    const bool single = (long long)b.max_new_len * G <= WAVE_ROWS;
    s.L.G = G;
    s.L.by_G = divisor_of(G);
    s.L.by_kv_heads = divisor_of(b.num_kv_heads);
    // the most that 32 rows look at
    const long long span = std::min((long long)b.max_pages * b.page_size, (long long)w.window + w.sinks + WAVE_ROWS / G + 1);
    const bool lengthy = (span + 63) / 64 >= LONG_TILES;
    const long long least_units = std::max<long long>((rows + 127) / 128, std::min(b.num_reqs, b.total_new_tokens)) * b.num_kv_heads;
    if (!single && least_units >= ROWS_UNITS) {
        s.rows_waves = lengthy ? 8 : 4;
        const int tile_rows = 32 * s.rows_waves, slots = 256 / s.rows_waves;
        const bool uniform = (long long)b.num_reqs * b.max_new_len == b.total_new_tokens;
        long long units = (rows / tile_rows + b.num_reqs) * b.num_kv_heads;
        if (uniform) units = ((long long)b.max_new_len * G + tile_rows - 1) / tile_rows * b.num_reqs * b.num_kv_heads;
        s.L.most_parts = units <= (lengthy ? (long long)CUT_ROUNDS * slots : PLACES / 4) * NUM_XCD ? (int)std::min((long long)MOST_PARTS, (span + 63) / 64 / MIN_TILES) : 1;
        if (s.L.most_parts < (lengthy ? 2 : 4)) s.L.most_parts = 1;
        if (uniform) {                                       // the plans are known: is any unit cut?
            auto cut = [&](long long n) {
                const long long rem = n % slots;
                return rem > 0 && rem <= slots / 2 && std::min<long long>(PLACES / rem, s.L.most_parts) >= (lengthy ? 2 : 4);
            };
            if (!cut(units / NUM_XCD) && !cut((units + NUM_XCD - 1) / NUM_XCD)) s.L.most_parts = 1;
        }
        s.grid = ((units + NUM_XCD - 1) / NUM_XCD + slots) * NUM_XCD;        // (units of the last round are `slots` workgroups at most)
        s.workspace = s.L.most_parts > 1 ? (size_t)NUM_XCD * PLACES * (lengthy ? Record<8>::FLOATS : Record<4>::FLOATS) * sizeof(float) : 0;
        return s;
    }
    const long long slots = single ? b.num_reqs : rows / WAVE_ROWS + b.num_reqs;
    s.L.slots = (int)slots;
    s.L.single = single;
    s.decode = single && b.max_new_len == 1 && G <= DECODE_ROWS;
    s.stream = s.decode && slots * b.num_kv_heads * span * (4 * D) > STREAM_BYTES;
    // as many parts as fill the chip, each of a tile for every wave at least
    const long long tiles = (span + 31) / 32, units = (single ? slots : std::max((rows + WAVE_ROWS - 1) / WAVE_ROWS, 1ll)) * b.num_kv_heads;
    s.L.parts = (int)std::max(1ll, std::min({COMPUTE_UNITS / units, (tiles + MIN_TILES - 1) / MIN_TILES, MOST_ITEMS / (slots * b.num_kv_heads)}));
    const long long items = slots * b.num_kv_heads * s.L.parts;
    s.L.items = (int)items;
    s.L.per_xcd = single ? 0 : (int)((items + NUM_XCD - 1) / NUM_XCD);
    s.L.by_slots = divisor_of((int)slots);
    s.L.by_parts = divisor_of(s.L.parts);
    s.grid = single ? items : (long long)s.L.per_xcd * NUM_XCD;
    s.workspace = s.L.parts > 1 ? (size_t)items * (s.decode ? DECODE_ROWS : WAVE_ROWS) * REC_STRIDE * sizeof(float) : 0;
    return s;
}

}  // namespace

size_t attn_window_workspace_bytes(const BatchView& b, const WindowView& w)
{
    return b.total_new_tokens == 0 || b.num_reqs == 0 ? 0 : deal_of(b, w).workspace;
}

hipError_t launch_attn_window(const AttnArgs& a, const WindowView& w, hipStream_t stream)
{
    const BatchView& b = a.b;
    const Deal s = deal_of(b, w);
    if (s.grid > 0x3fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)s.grid);
    if (s.rows_waves == 8) hipLaunchKernelGGL((attn_window_rows_kernel<8>), grid, dim3(64 * 8), 0, stream, a, w, s.L);
    else if (s.rows_waves == 4) hipLaunchKernelGGL((attn_window_rows_kernel<4>), grid, dim3(64 * 4), 0, stream, a, w, s.L);
    else if (s.stream) hipLaunchKernelGGL((attn_window_decode_kernel<true>), grid, dim3(64 * WAVES), 0, stream, a, w, s.L);
    else if (s.decode) hipLaunchKernelGGL((attn_window_decode_kernel<false>), grid, dim3(64 * WAVES), 0, stream, a, w, s.L);
    else hipLaunchKernelGGL(attn_window_keys_kernel, grid, dim3(64 * WAVES), 0, stream, a, w, s.L);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess || s.workspace == 0) return err;
    if (s.rows_waves > 0) {
        const dim3 merge(NUM_XCD * PLACES * SUB);
        if (s.rows_waves == 8) hipLaunchKernelGGL((attn_window_rows_merge_kernel<8>), merge, dim3(256), 0, stream, a, w, s.L);
        else hipLaunchKernelGGL((attn_window_rows_merge_kernel<4>), merge, dim3(256), 0, stream, a, w, s.L);
    } else {
        const int rows = (int)std::min<long long>((long long)b.max_new_len * s.L.G, WAVE_ROWS), groups = (rows + WAVES - 1) / WAVES;
        const dim3 merge((unsigned)(s.L.slots * b.num_kv_heads * groups));
        if (s.decode) hipLaunchKernelGGL((attn_window_merge_kernel<DECODE_ROWS>), merge, dim3(64 * WAVES), 0, stream, a, w, s.L, groups);
        else hipLaunchKernelGGL((attn_window_merge_kernel<WAVE_ROWS>), merge, dim3(64 * WAVES), 0, stream, a, w, s.L, groups);
    }
    return hipGetLastError();
}

}  // namespace emm
