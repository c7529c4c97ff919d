// Attention of many rows over the 8-bit cache: prompts and longer chunks (formulas: include/emm_fp8.h).
//
// Bound by the matrix pipe and the instructions around it.  Rows are (new token, query head of a KV group) pairs of one
// (request, KV head), token-major; a workgroup of 8 waves takes 256 of them (a unit), a wave 32, and streams the keys
// in tiles of 64, each fetched once for the workgroup:
// K and V go to LDS as they are (K three tiles ahead, V two), and from there through the wave that fetched them, which makes
// them bf16 in their keys' scales (exact) and puts them into rings of two tiles, in 16-byte chunks placed so that no read of
// them meets a bank twice.  (The stores do, 8 % of the cycles; storing the halves the other way round in every second four lanes
// ends that and changes no time.)  Scale bytes travel with them, K's a tile earlier: a wave brings those of other waves' rows, and K
// is converted before the barrier that V waits for.  (Each wave converting what it needs of K in its registers takes 64 conversions
// a tile in place of 8: two chunks of 2048 behind 16 k 923 us, so 900.)
// S^T = K Q^T and O^T += V^T P^T are v_mfma_f32_32x32x16_bf16.  A lane has one row and 32 of a tile's keys; K's rows lie in
// LDS such that its weights, rounded to bf16, are the second product's operand as they are, and which channels a step of the first
// takes is the same for K and q.
// Weights are exp2(S c - m) with a reference m that is the row's maximum over its first tile, and follows only where the
// weights that a lane has of half a tile (16 keys; its partner lane has the row's other 16) sum to more than 2^20: any reference gives the
// same result as long as the sums stay finite, which emm_fp8.h says of what values they do, and the sum, which is taken before the weights are
// used, tells in time.  So the loop takes no maxima.  Row sums are of the weights before they are rounded (of the rounded ones, and lse
// with them, they would be off by up to 2^-8 where few keys count).  The product's are rounded to bf16 because it takes both operands so; in
// 32 bits it would need 16 times the matrix instructions.  out is then 0.0022 of itself off (root mean square) where its own rounding makes 0.0017.
//
// Measured (28 query heads over 4 KV heads): two chunks of 2048 behind 16384 890 to 960 us on different cards, 1070 to 1150 TFLOP/s, where
// a large bf16 matrix product reaches 1346; the matrix units are busy 61 % of the cycles, at 1.9 of 2.4 GHz: it is the power that ends
// there (a last round spread evenly over all compute units in place of three quarters of them took as long).  Eight chunks of 128 to
// 512 behind an image 65.3 us, of which 6 are the merge; 36 tokens behind 16384 28.2 us: 64 pieces, four tiles each, of which four are
// what a piece costs before its first tile (lengths, pages, rows of q, tiles: dependent trips), 8.5 the records' way through memory.
#include <algorithm>
#include <type_traits>

#include "attn_fp8_common.h"

namespace emm {

namespace {

using namespace fp8;
using bf16attn::lds_dma16;
using bf16attn::swap23;
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int NW = 8;                                    // waves of a workgroup
constexpr int BR = 32 * NW;                              // rows of a unit
constexpr int BC = 64;                                   // keys of a tile
constexpr int PLACES = 256;                              // workgroups that run at once: one on each compute unit
constexpr int MAX_PARTS = 128;                           // pieces of a unit (one unit of 30 k keys 24.3 us; 64: 26.0, 256: 28.4)
constexpr int MIN_TILES_ALONE = 2, MIN_TILES_BEHIND = 4;    // key tiles of a piece where no unit is whole (16 units of 1000 keys 18.8 us; 3: 19.2, 4: 20.0), and
                                                            // behind whole ones (8 images' chunks 65.3; 2: 67.1, 8: 68.6)
constexpr float LAG_LIMIT = 1048576.f;                   // 2^20 for 16 keys: 2^16 a key, the factor in the header's bound on V
constexpr int QK_OPS = 80;                               // of a tile's 119 softmax instructions beside the score products (72, 88: 1 % slower; at least 63)

// LDS
constexpr int TILE = BC * HEAD_DIM * 2, RAW_TILE = BC * HEAD_DIM;
constexpr int K_AT = 0, V_AT = K_AT + 2 * TILE, K_RAW_AT = V_AT + 2 * TILE, RAW_AT = K_RAW_AT + 4 * RAW_TILE, S_AT = RAW_AT + 2 * RAW_TILE, FLAG_AT = S_AT + 4 * 128, SMEM = FLAG_AT + 64;
constexpr int OUT_STRIDE = 272;                          // bytes between output rows on their way out
static_assert(NW * 32 * OUT_STRIDE <= FLAG_AT, "output rows are staged over the rings");
constexpr int FETCHES = 3;                               // of a wave for a tile: K, V, scales

constexpr int RECORD_FLOATS = (64 + 2) * 64 * NW;        // of a piece: 64 accumulators of each thread in groups of four, then m and l
constexpr int TEAMS = 4;                                 // waves of the merge,
constexpr int MERGERS = 1024;                            // and its workgroups at most
constexpr int FEW_UNITS = 8;                             // units that give the merge too little to do with 32 channels at a time

// how the units of a batch are laid out over the grid
struct Layout {
    int units_max;          // units of the batch at most, rounded up to 8
    int cut;                // 1: units behind the last full round of PLACES may be cut along the keys
    int G;
    Divisor by_G, by_kv_heads;
};

struct Unit {
    int req, kvh, tile;     // req < 0: nothing to do
    int new_len, prefix_len, cu_new;
    int parts, part, slot;  // planned pieces of the unit, which one, and the unit's place among those that are cut
};

// Units in order: requests, in a request row tiles from the last (which sees the most keys) to the first, of a row tile the
// KV heads; neighbouring workgroups run on neighbouring XCDs, so an XCD has the same few heads throughout and their K and V
// go through its L2.  Whole rounds of PLACES units first; the rest, if few, are cut in as many pieces as fill the chip.
struct Plan {
    const BatchView& b;
    const Layout& L;
    int lane, new_lane, prefix_lane, cu_lane, incl;      // of the 64 requests looked at
    int total;                                           // row tiles of the batch
    int units, full, rest, parts;                        // full: units in whole rounds; rest: those behind, in so many pieces each

    __device__ int look(int first)                       // lane's request first + lane; returns the row tiles of the 64
    {
        const int r = min(first + lane, b.num_reqs - 1);
        new_lane = b.new_lens[r];
        prefix_lane = b.prefix_lens[r];
        cu_lane = b.cu_new_lens[r];
        const int n = first + lane < b.num_reqs ? clamp_new_len(b, new_lane, false) : 0;
        incl = scan64((n * L.G + BR - 1) / BR);
        return __builtin_amdgcn_readlane(incl, 63);
    }
    __device__ Plan(const BatchView& batch, const Layout& layout) : b(batch), L(layout), lane(threadIdx.x & 63), total(0)
    {
        for (int first = 0; first < b.num_reqs; first += 64) total += look(first);
        units = total * b.num_kv_heads;
        full = L.cut ? units / PLACES * PLACES : units;
        rest = units - full;
        parts = rest == 0 ? 1 : min(PLACES / rest, MAX_PARTS);
    }
    __device__ Unit unit(int ordinal)
    {
        Unit u;
        u.req = -1;
        u.parts = ordinal < full ? 1 : parts;
        u.part = 0;
        u.slot = ordinal - full;
        if (ordinal >= units) return u;
        const int nth = L.by_kv_heads.quotient(ordinal); // row tile of the batch
        u.kvh = ordinal - nth * b.num_kv_heads;
        int before = 0;
        for (int first = 0; first < b.num_reqs; first += 64) {
            const int sum = b.num_reqs <= 64 ? total : look(first);
            if (nth < before + sum) {
                const unsigned long long hit = __builtin_amdgcn_ballot_w64(incl > nth - before);
                const int at = __builtin_ctzll(hit);
                u.req = first + at;
                u.tile = __builtin_amdgcn_readlane(incl, at) - 1 - (nth - before);
                u.new_len = __builtin_amdgcn_readlane(new_lane, at);
                u.prefix_len = __builtin_amdgcn_readlane(prefix_lane, at);
                u.cu_new = __builtin_amdgcn_readlane(cu_lane, at);
                return u;
            }
            before += sum;
        }
        return u;
    }
    __device__ Unit of_workgroup(int wg)
    {
        if (wg < full || rest == 0) return unit(wg);
        const int part = (wg - full) / rest;
        Unit u = unit(part < parts ? wg - part * rest : units);
        u.part = part;
        return u;
    }
};

// the first of a unit's key tiles that is piece `part`'s (part == pieces: behind the last); without a sign, since
// MAX_PARTS times the tiles of the longest context is 2^31
constexpr int piece_begin(int part, int n_tiles, int pieces) { return (int)((uint32_t)part * (uint32_t)n_tiles / (uint32_t)pieces); }
static_assert(MAX_PARTS * (MOST_SLOTS / BC) < 1ll << 32 && piece_begin(MAX_PARTS, MOST_SLOTS / BC, MAX_PARTS) == MOST_SLOTS / BC, "a piece's end holds in 32 bits");

// a unit's rows and keys
struct Extent {
    int N, P, first_row, ctx, n_rows, row0, kv_len, n_tiles, pieces;
};
template <bool CAUSAL>
__device__ inline Extent extent_of(const BatchView& b, const Layout& L, const Unit& u, bool alone)
{
    Extent e;
    e.N = clamp_new_len(b, u.new_len, CAUSAL);
    e.n_rows = e.N * L.G;
    e.row0 = u.tile * BR;
    e.P = clamp_prefix_len(b, u.prefix_len, CAUSAL ? e.N : 0);
    e.first_row = clamp_first_row(b, u.cu_new, e.N);
    e.ctx = CAUSAL ? e.P + e.N : e.P;
    e.kv_len = CAUSAL ? e.P + L.by_G.quotient(min(e.row0 + BR, e.n_rows) - 1) + 1 : e.P;
    e.n_tiles = (e.kv_len + BC - 1) / BC;
    e.pieces = min(u.parts, max(1, e.n_tiles / (alone ? MIN_TILES_ALONE : MIN_TILES_BEHIND)));
    return e;
}

__device__ inline void lds_dma4(const void* base, uint32_t byte_offset, uint32_t lds_byte_offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds_byte_offset), "v"(byte_offset), "s"(base) : "memory");
}
__device__ inline void pin(float& x) { asm volatile("" : "+v"(x)); }
__device__ inline void pin(bf16x2& x)
{
    uint32_t u = __builtin_bit_cast(uint32_t, x);
    asm volatile("" : "+v"(u));
    x = __builtin_bit_cast(bf16x2, u);
}
template <int BEGIN, int END, class F>
__device__ inline void static_for(F&& f)
{
    if constexpr (BEGIN < END) {
        f(std::integral_constant<int, BEGIN>{});
        static_for<BEGIN + 1, END>(f);
    }
}

template <bool CAUSAL>
__global__ __launch_bounds__(64 * NW, 2) void attn_fp8_tiles_kernel(AttnFp8Args a, Layout L)
{
    __shared__ __attribute__((aligned(1024))) unsigned char smem[SMEM];
    const BatchView& b = a.b;
    const Unit u = Plan(b, L).of_workgroup(blockIdx.x);
    if (u.req < 0) return;
    const Extent e = extent_of<CAUSAL>(b, L, u, L.units_max <= PLACES);
    if (e.row0 >= e.n_rows || u.part >= e.pieces) return;
    const int t_begin = piece_begin(u.part, e.n_tiles, e.pieces), n_tiles = piece_begin(u.part + 1, e.n_tiles, e.pieces) - t_begin;

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int l32 = lane & 31, h32 = lane >> 5;
    const int wrow0 = e.row0 + wave * 32;
    const bool active = wrow0 < e.n_rows;                    // a wave without rows fetches its share and meets the others
    const int row = min(wrow0 + l32, e.n_rows - 1), tok = L.by_G.quotient(row);
    const int limit = CAUSAL ? e.P + tok : e.P - 1;          // last key that the lane's row sees
    const int wave_clear = CAUSAL ? (e.P + L.by_G.quotient(min(wrow0, e.n_rows - 1)) + 1) / BC : e.P / BC;    // tiles that all rows of the wave see whole,
    const int unit_clear = CAUSAL ? (e.P + L.by_G.quotient(e.row0) + 1) / BC : e.P / BC;                      // and of the unit

    // ---- fetches.  Wave w brings rows 8 w .. 8 w + 7 of a tile, of 16-key block 4 tile + w / 2 (1 KB of K and of V), and that block's
    //      16 scale bytes of K (even waves) or V (odd).
    const int32_t* __restrict__ pt = b.page_table + (long long)u.req * b.max_pages;
    const int n_blocks = (e.ctx + 15) >> 4;
    const uint32_t smem_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
    const int r16 = 8 * (wave & 1) + (lane >> 3);            // row in the block
    const uint32_t k_src = swap23(r16) * HEAD_DIM + ((lane & 7) << 4);    // K: LDS row = block row with the key's bits 2 and 3 changed places
    const uint32_t v_src = (wave & 1) * 1024 + lane * 16;    // V: as it is
    const unsigned char* scales = (wave & 1) ? a.pools.v_scale : a.pools.k_scale;
    int block_ids = 0, ids_from = 0;                         // lane k: the wave's block of tile ids_from + k, in blocks of the pool
    auto ask_blocks = [&](int from) {
        const int blk = min(4 * (from + lane) + (wave >> 1), n_blocks - 1);
        const int page = min(max(pt[blk >> b.page_shift], 0), b.num_pages - 1);
        block_ids = ((page * b.num_kv_heads + u.kvh) << b.page_shift) + (blk & ((1 << b.page_shift) - 1));
        ids_from = from;
    };
    if (n_tiles > 0) ask_blocks(t_begin);
    // q's rows travel with the block ids; 64 channels a lane: 64 s + 32 h32 + 0 .. 31
    uint32_t pairs[32];
    {
        const __bf16* qp = (const __bf16*)a.q + ((long long)(e.first_row + tok) * b.num_q_heads + u.kvh * L.G + row - tok * L.G) * HEAD_DIM + 32 * h32;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint4 x = *(const uint4*)(qp + 64 * (i >> 2) + 8 * (i & 3));
            pairs[4 * i] = x.x; pairs[4 * i + 1] = x.y; pairs[4 * i + 2] = x.z; pairs[4 * i + 3] = x.w;
        }
    }
    auto block_of = [&](int t) { return (long long)__builtin_amdgcn_readlane(block_ids, t - ids_from); };
    auto fetch_k = [&](int t, int slot) { lds_dma16(a.pools.k + block_of(t) * 2048, k_src, smem_base + K_RAW_AT + slot * RAW_TILE + wave * 1024); };
    auto fetch_v = [&](int t, int slot) { lds_dma16(a.pools.v + block_of(t) * 2048, v_src, smem_base + RAW_AT + slot * RAW_TILE + wave * 1024); };
    const int k_scales = 1 - (wave & 1);                     // the wave brings scales of K, and those a tile earlier
    auto fetch_scales = [&](int t, int slot) {
        const unsigned char* src = scales + block_of(t) * 16;
        if (lane < 4) lds_dma4(src, lane * 4, smem_base + S_AT + slot * 128 + (wave & 1) * 64 + (wave >> 1) * 16);
    };

    // ---- K to bf16: 16 channels of a key per lane.  K tile: chunk c of 16 bytes of row r lies at place c ^ (r mod 16)
    const int k_row = 8 * wave + (lane >> 3), k_wr = K_AT + k_row * 256 + (((2 * (lane & 7)) ^ (k_row & 15)) << 4), ks_rd = S_AT + 16 * (wave >> 1) + swap23(r16);
    auto read_raw_k = [&](int slot) -> uint4 { return *(const uint4*)(smem + K_RAW_AT + slot * RAW_TILE + wave * 1024 + lane * 16); };
    auto store_k = [&](const uint4& codes, int scale, int slot) {
        const float s = up_scale(scale);
        auto half = [&](uint32_t w0, uint32_t w1) -> uint4 {
            auto pair = [&](uint32_t w, auto upper) -> uint32_t { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, decltype(upper)::value)); };
            return make_uint4(pair(w0, std::false_type{}), pair(w0, std::true_type{}), pair(w1, std::false_type{}), pair(w1, std::true_type{}));
        };
        *(uint4*)(smem + slot * TILE + k_wr) = half(codes.x, codes.y);
        *(uint4*)(smem + slot * TILE + (k_wr ^ 16)) = half(codes.z, codes.w);
    };

    // ---- V to bf16: 16 channels of a key per lane.  Keys behind the context hold anything: zeros in their place.  In tiles that not every
    //      row sees whole, a NaN would reach rows that do not see it (0 * NaN): it becomes a zero too, and flags say that there was one.
    const int v_key = 8 * wave + (lane >> 3);
    // V tile: chunk c of 16 bytes of key k lies at place c ^ 4 (k mod 4) ^ (k mod 2): the transposing reads meet no bank twice
    const int v_wr = V_AT + v_key * 256 + (((2 * (lane & 7)) ^ ((v_key & 3) << 2) ^ (v_key & 1)) << 4);
    uint4 raw;
    int raw_scale;
    auto read_raw = [&](int raw_slot, int s_slot) {
        raw = *(const uint4*)(smem + RAW_AT + raw_slot * RAW_TILE + wave * 1024 + lane * 16);
        raw_scale = smem[S_AT + s_slot * 128 + 64 + v_key];
    };
    auto check_raw = [&](int t, int v_slot) {                // tiles from unit_clear on
        if (t * BC + v_key >= e.ctx) {
            raw = make_uint4(0, 0, 0, 0);
            raw_scale = BIAS;
        }
        if constexpr (CAUSAL) {
            const uint32_t n0 = nan_bytes(raw.x), n1 = nan_bytes(raw.y), n2 = nan_bytes(raw.z), n3 = nan_bytes(raw.w);
            const bool any = __builtin_amdgcn_ballot_w64((n0 | n1 | n2 | n3) != 0) != 0;
            if (any) raw = make_uint4(raw.x & ~((n0 >> 7) * 0xffu), raw.y & ~((n1 >> 7) * 0xffu), raw.z & ~((n2 >> 7) * 0xffu), raw.w & ~((n3 >> 7) * 0xffu));
            if (lane == 0) smem[FLAG_AT + 8 * v_slot + wave] = any ? 1 : 0;
        }
    };
    auto widen = [&](int half) -> uint4 {                    // 8 channels: the lower or upper half
        const float s = up_scale(raw_scale);
        const uint32_t w0 = half ? raw.z : raw.x, w1 = half ? raw.w : raw.y;
        const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, false), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, true);
        const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, false), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, true);
        return make_uint4(__builtin_bit_cast(uint32_t, p0), __builtin_bit_cast(uint32_t, p1), __builtin_bit_cast(uint32_t, p2), __builtin_bit_cast(uint32_t, p3));
    };
    auto store_v = [&](int v_slot) {
        *(uint4*)(smem + v_slot * TILE + v_wr) = widen(0);
        *(uint4*)(smem + v_slot * TILE + (v_wr ^ 16)) = widen(1);
    };

    // which of the lane's 64 outputs meet a NaN of V: bit 4 (4 nb + v / 4) + v % 4.  Rare: from global memory, key by key.
    unsigned long long poison = 0;
    auto find_poison = [&](int t) {
        for (int k = 0; k < BC; ++k) {
            const int key = t * BC + k;
            if (key >= e.ctx) break;
            const int page = min(max(pt[(key >> 4) >> b.page_shift], 0), b.num_pages - 1);
            const long long pool_row = ((((long long)page * b.num_kv_heads + u.kvh) << b.page_shift) + ((key >> 4) & ((1 << b.page_shift) - 1))) * 16 + (key & 15);
            const uint32_t* codes = (const uint32_t*)(a.pools.v + pool_row * HEAD_DIM) + h32;
            for (int c = 0; c < 16; ++c) {
                const uint32_t n = nan_bytes(codes[2 * c]) >> 7;
                const unsigned long long bits = (n | n >> 7 | n >> 14 | n >> 21) & 15u;
                if (key <= limit) poison |= bits << (4 * c);
            }
        }
    };

    // ---- operands
    const int k_rd = K_AT + l32 * 256 + (((4 * h32) ^ (l32 & 15)) << 4);
    auto read_k = [&](int slot, int kb, int j) -> bf16x8 {       // 8 of the lane's 64 channels of a key, as q_operand(j)
        return *(const bf16x8*)(smem + slot * TILE + kb * 32 * 256 + (k_rd ^ (((j >> 2) * 8 + (j & 3)) << 4)));
    };
    // within each 16 lanes, lane j gives the address of 4 channels of key k0 + j / 4 and gets keys k0 .. k0 + 3 of channel d0 + j
    const int v_rd = V_AT + (8 * h32 + ((lane & 15) >> 2)) * 256 + ((4 * ((lane & 15) >> 2) + 2 * ((lane >> 4) & 1) + (((lane & 3) >> 1) ^ ((lane >> 2) & 1))) << 4) + (lane & 1) * 8;
    auto read_v = [&](int slot, int k16, int nb) -> bf16x8 {     // keys 16 k16 .. + 15, channels 32 nb .. + 31
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        const unsigned char* src = smem + slot * TILE + 16 * k16 * 256 + (v_rd ^ (nb << 6));
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src + 4 * 256));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto q_operand = [&](int j) -> bf16x8 { return __builtin_bit_cast(bf16x8, u32x4{pairs[4 * j], pairs[4 * j + 1], pairs[4 * j + 2], pairs[4 * j + 3]}); };
    const float c_log2 = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, b.softmax_scale * LOG2E)));

    f32x16 o[4];
    float m = 0.f, l = 0.f;
#pragma unroll
    for (int nb = 0; nb < 4; ++nb)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[nb][v] = 0.f;

    // register v of block kb is key 32 kb + 16 (v / 8) + 8 h32 + v % 8 of the tile
    auto mask_tile = [&](int t, f32x16 (&s)[2]) {
        const int last = limit - 8 * h32 - t * BC;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (32 * kb + 16 * (v >> 3) + (v & 7) > last) s[kb][v] = -INFINITY;
    };
    auto row_max = [&](const f32x16 (&s)[2]) -> float {
        float x = s[0][0];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) x = fmaxf(x, s[kb][v]);
        return pair_max(x);
    };
    auto scores = [&](int slot, f32x16 (&s)[2]) {            // not interleaved: first and only tiles
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int v = 0; v < 16; ++v) s[kb][v] = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_k(slot, kb, j), q_operand(j), s[kb], 0, 0, 0);
        }
    };
    // weights of half a tile (32 keys), packed, and their sum over the lane's keys
    auto weights = [&](const f32x16& s, uint32_t* p) -> float {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            bf16x2 w;
            const float x = __builtin_amdgcn_exp2f(fmaf(s[2 * i], c_log2, -m)), y = __builtin_amdgcn_exp2f(fmaf(s[2 * i + 1], c_log2, -m));
            sum += x + y;
            w[0] = (__bf16)x;
            w[1] = (__bf16)y;
            p[i] = __builtin_bit_cast(uint32_t, w);
        }
        return sum;
    };
    // The weights of a half, which sum to `sum`, are about to be used: where they have outgrown the reference it becomes the row's
    // maximum so far, and they are made again; and where it has changed since they were made from `ref`.
    auto settle = [&](const f32x16& s, uint32_t* p, float sum, float ref) {
        const bool grown = sum > LAG_LIMIT;
        if (__builtin_amdgcn_ballot_w64(grown || m != ref) != 0) {
            // (both lanes of a row decide alike)
            if (pair_max(sum) > LAG_LIMIT) {
                float top = s[0];
#pragma unroll
                for (int v = 1; v < 16; ++v) top = fmaxf(top, s[v]);
                const float to = fmaxf(m, pair_max(top) * c_log2), scale = __builtin_amdgcn_exp2f(m - to);
                m = to;
                l *= scale;
#pragma unroll
                for (int nb = 0; nb < 4; ++nb)
#pragma unroll
                    for (int v = 0; v < 16; ++v) o[nb][v] *= scale;
            }
            if (m != ref) sum = weights(s, p);
        }
        l += sum;
    };
    auto p_operand = [&](const uint32_t* p, int k16) -> bf16x8 {
        return __builtin_bit_cast(bf16x8, u32x4{p[4 * k16], p[4 * k16 + 1], p[4 * k16 + 2], p[4 * k16 + 3]});
    };
    auto flagged = [&](int v_slot) -> bool {
        typedef int i32x2 __attribute__((ext_vector_type(2)));
        const i32x2 f = *(const i32x2*)(smem + FLAG_AT + 8 * v_slot);
        return __builtin_amdgcn_readfirstlane(f[0] | f[1]) != 0;
    };

    if (n_tiles > 0) {
        // (q is waited for here, before the fetches: behind them it would be waited for with them)
        __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0)
#pragma unroll
        for (int i = 0; i < 32; ++i) asm volatile("" : "+v"(pairs[i]));
        fetch_k(t_begin, 0);
        fetch_v(t_begin, 0);
        fetch_scales(t_begin, 0);
        if (n_tiles > 1) {
            fetch_k(t_begin + 1, 1);
            fetch_v(t_begin + 1, 1);
            fetch_scales(t_begin + 1, 1);
            fetch_k(t_begin + 2, 2);
            fetch_scales(t_begin + 2, 2);
            if (k_scales) fetch_scales(t_begin + 3, 3);
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0)
        __syncthreads();
        read_raw(0, 0);
        if (t_begin >= unit_clear) check_raw(t_begin, 0);
        store_v(0);
        store_k(read_raw_k(0), smem[ks_rd], 0);
        if (n_tiles > 1) store_k(read_raw_k(1), smem[ks_rd + 128], 1);
        __syncthreads();
        const int t_end = t_begin + n_tiles;
        if (!active) {
            if (n_tiles > 1) __syncthreads();
            for (int i = t_begin; i + 1 < t_end; ++i) {
                const int R = (i - t_begin) & 3;
                if (i + 4 - ids_from >= 64) ask_blocks(i + 2);
                fetch_k(i + 3, (R + 3) & 3);
                fetch_v(i + 2, R & 1);
                fetch_scales(i + 3 + k_scales, (R + 3 + k_scales) & 3);
                __builtin_amdgcn_s_waitcnt(0x0f70 | FETCHES);
                __builtin_amdgcn_sched_barrier(0);
                store_k(read_raw_k((R + 2) & 3), smem[ks_rd + ((R + 2) & 3) * 128], R & 1);
                __syncthreads();
                read_raw((R + 1) & 1, (R + 1) & 3);
                if (i + 1 >= unit_clear) check_raw(i + 1, (R + 1) & 1);
                store_v((R + 1) & 1);
            }
            __syncthreads();
        } else {
            f32x16 sc[2][2];                                 // scores of tile i in sc[i & 1]
            scores(0, sc[0]);
            if (n_tiles > 1) __syncthreads();                // (tile 2 goes where tile 0 was)
            if (t_begin >= wave_clear) mask_tile(t_begin, sc[0]);
            const float top = row_max(sc[0]) * c_log2;
            m = top > -INFINITY ? top : 0.f;                 // (a row that sees none of a piece's keys: its weights are zeros)

            // Iteration i: scores of tile i + 1 and the weights of tile i; then everybody's fetches for the next tiles are published;
            // then the values of tile i, and V of tile i + 1 to bf16.
            auto iteration = [&](int i, auto par) {
                constexpr int R = decltype(par)::value;
                constexpr int KS = (R + 1) & 3, VS = R & 1, VN = (R + 1) & 1;
                f32x16 (&s_cur)[2] = sc[R & 1];
                f32x16 (&s_nxt)[2] = sc[(R & 1) ^ 1];
                uint32_t p[16];
                float fa[16], fb[16], ea[16], eb[16], sums[4] = {};
                const float ref = m;
                // pair g: F F (scale, subtract), E E (exp2), A A (sums), C (round): a stream in which nothing follows what it depends on
                auto softmax_op = [&](auto idx_c) {
                    constexpr int idx = decltype(idx_c)::value, g = idx / 7, slot = idx % 7;
                    if constexpr (slot == 0 && g < 16) {
                        ea[g] = __builtin_amdgcn_exp2f(fa[g]);
                        pin(ea[g]);
                    } else if constexpr (slot == 1 && g < 16) {
                        eb[g] = __builtin_amdgcn_exp2f(fb[g]);
                        pin(eb[g]);
                    } else if constexpr (slot == 2 && g >= 1) {
                        bf16x2 w;
                        w[0] = (__bf16)ea[g - 1];
                        w[1] = (__bf16)eb[g - 1];
                        pin(w);
                        p[g - 1] = __builtin_bit_cast(uint32_t, w);
                    } else if constexpr (slot == 3 && g + 1 < 16) {
                        fa[g + 1] = fmaf(s_cur[(g + 1) >> 3][2 * ((g + 1) & 7)], c_log2, -ref);
                        pin(fa[g + 1]);
                    } else if constexpr (slot == 4 && g + 1 < 16) {
                        fb[g + 1] = fmaf(s_cur[(g + 1) >> 3][2 * ((g + 1) & 7) + 1], c_log2, -ref);
                        pin(fb[g + 1]);
                    } else if constexpr (slot == 5 && g >= 1) {
                        sums[2 * ((g - 1) >> 3)] += ea[g - 1];
                        pin(sums[2 * ((g - 1) >> 3)]);
                    } else if constexpr (slot == 6 && g >= 1) {
                        sums[2 * ((g - 1) >> 3) + 1] += eb[g - 1];
                        pin(sums[2 * ((g - 1) >> 3) + 1]);
                    }
                };
                __builtin_amdgcn_s_setprio(0);
                constexpr int OPS = 17 * 7, OPS_HERE = QK_OPS;   // (pairs 0 .. 7, the first half, are done after 63)
                fa[0] = fmaf(s_cur[0][0], c_log2, -ref);
                fb[0] = fmaf(s_cur[0][1], c_log2, -ref);
                bf16x8 ka[16 + 2];
                ka[0] = read_k(VN, 0, 0);
                ka[1] = read_k(VN, 1, 0);
                uint4 raw_k;
                int raw_k_scale;
                __builtin_amdgcn_sched_barrier(0);
                static_for<0, 16>([&](auto kc) {
                    constexpr int k = decltype(kc)::value, kb = k & 1;
                    if constexpr (k + 2 < 16) ka[k + 2] = read_k(VN, k & 1, (k + 2) >> 1);
                    if constexpr (k < 2) {
                        f32x16 zero;
#pragma unroll
                        for (int v = 0; v < 16; ++v) zero[v] = 0.f;
                        s_nxt[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[k], q_operand(0), zero, 0, 0, 0);
                    } else {
                        s_nxt[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[k], q_operand(k >> 1), s_nxt[kb], 0, 0, 0);
                    }
                    static_for<(k * OPS_HERE) / 16, ((k + 1) * OPS_HERE) / 16>(softmax_op);
                    if constexpr (k == 2) fetch_k(i + 3, (R + 3) & 3);
                    if constexpr (k == 4) fetch_v(i + 2, R & 1);
                    if constexpr (k == 6) fetch_scales(i + 3 + k_scales, (R + 3 + k_scales) & 3);
                    if constexpr (k == 10) {
                        __builtin_amdgcn_s_waitcnt(0x0f70 | FETCHES);        // all fetches but this iteration's have landed
                        __builtin_amdgcn_sched_barrier(0);
                        raw_k = read_raw_k((R + 2) & 3);
                        raw_k_scale = smem[ks_rd + ((R + 2) & 3) * 128];
                    }
                    if constexpr (k == 14) store_k(raw_k, raw_k_scale, R & 1);
                    __builtin_amdgcn_sched_barrier(0);
                });
                settle(s_cur[0], p, sums[0] + sums[1], ref);
                __syncthreads();
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(1);                       // a wave at its value products, which have less beside them, goes first
                read_raw(VN, KS);
                bf16x8 vf[16 + 2];
                vf[0] = read_v(VS, 0, 0);
                vf[1] = read_v(VS, 0, 1);
                if (CAUSAL && i >= unit_clear) {
                    if (flagged(VS)) find_poison(i);
                }
                if (i + 1 >= unit_clear) check_raw(i + 1, VN);
                __builtin_amdgcn_sched_barrier(0);
                static_for<0, 16>([&](auto kc) {
                    constexpr int k = decltype(kc)::value;
                    if constexpr (k + 2 < 16) vf[k + 2] = read_v(VS, (k + 2) >> 2, (k + 2) & 3);
                    if constexpr (k == 8) {
                        settle(s_cur[1], p + 8, sums[2] + sums[3], ref);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    o[k & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k], p_operand(p, k >> 2), o[k & 3], 0, 0, 0);
                    if constexpr (k < 8) static_for<OPS_HERE + (k * (OPS - OPS_HERE)) / 8, OPS_HERE + ((k + 1) * (OPS - OPS_HERE)) / 8>(softmax_op);
                    if constexpr (k == 10) store_v(VN);
                    if constexpr (k == 12) {
                        if (i + 1 >= wave_clear) {
                            __builtin_amdgcn_sched_barrier(0);
                            mask_tile(i + 1, s_nxt);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
            };
            int i = t_begin;
            for (;;) {
                if (i + 7 - ids_from >= 64) ask_blocks(i + 2);       // tiles i + 2 .. i + 7 may be fetched in this trip
                if (i + 1 >= t_end) break;
                iteration(i, std::integral_constant<int, 0>{});
                if (i + 2 >= t_end) break;
                iteration(i + 1, std::integral_constant<int, 1>{});
                if (i + 3 >= t_end) break;
                iteration(i + 2, std::integral_constant<int, 2>{});
                if (i + 4 >= t_end) break;
                iteration(i + 3, std::integral_constant<int, 3>{});
                i += 4;
            }
            // the last tile, a half at a time: the first half's values are taken before the second half may raise the reference
            const int odd = (n_tiles - 1) & 1;
            __syncthreads();
            if (CAUSAL && t_end - 1 >= unit_clear) {
                if (flagged(odd)) find_poison(t_end - 1);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t p[8];
                const float ref = m;
                if (odd) settle(sc[1][h], p, weights(sc[1][h], p), ref);
                else settle(sc[0][h], p, weights(sc[0][h], p), ref);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    o[k & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_v(odd, 2 * h + (k >> 2), k & 3), p_operand(p, k >> 2), o[k & 3], 0, 0, 0);
            }
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);                  // the last fetches have landed, and
        __syncthreads();                                     // all are past their reads: the rings are free
    }
    if (!active) return;
    if (CAUSAL && __builtin_amdgcn_ballot_w64(poison != 0) != 0) {
#pragma unroll
        for (int nb = 0; nb < 4; ++nb)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if ((poison >> (16 * nb + v)) & 1) o[nb][v] = __builtin_nanf("");
    }
    const float l_row = pair_sum(l);
    if (e.pieces > 1) {
        float* rec = (float*)a.workspace + (long long)(u.slot * u.parts + u.part) * RECORD_FLOATS;
#pragma unroll
        for (int g = 0; g < 16; ++g)
            *(f32x4*)(rec + (g * 64 * NW + tid) * 4) = f32x4{o[g >> 2][4 * (g & 3)], o[g >> 2][4 * (g & 3) + 1], o[g >> 2][4 * (g & 3) + 2], o[g >> 2][4 * (g & 3) + 3]};
        *(f32x2*)(rec + 64 * 64 * NW + 2 * tid) = f32x2{l_row == 0.f ? -INFINITY : m, l_row};
        return;
    }
    // rows go out through LDS, so that a store writes four whole rows
    const float inv = l_row == 0.f ? 0.f : 1.0f / l_row;
    unsigned char* stage = smem + wave * (32 * OUT_STRIDE);
#pragma unroll
    for (int g = 0; g < 16; ++g) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 w;
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = (__bf16)(o[g >> 2][4 * (g & 3) + k] * inv);
        *(bf16x4*)(stage + l32 * OUT_STRIDE + 2 * (32 * (g >> 2) + 8 * (g & 3) + 4 * h32)) = w;
    }
    auto place_of = [&](int r) -> long long {
        const int t = L.by_G.quotient(r);
        return (long long)(e.first_row + t) * b.num_q_heads + u.kvh * L.G + r - t * L.G;
    };
    if (a.lse != nullptr && h32 == 0 && wrow0 + l32 < e.n_rows) a.lse[place_of(wrow0 + l32)] = l_row == 0.f ? -INFINITY : (m + log2f(l_row)) * LN2;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r = 4 * j + (lane >> 4);
        if (wrow0 + r < e.n_rows)
            *(uint4*)((__bf16*)a.out + place_of(wrow0 + r) * HEAD_DIM + (lane & 15) * 8) = *(const uint4*)(stage + r * OUT_STRIDE + (lane & 15) * 16);
    }
}

// The pieces of the units that were cut; bound by their records, 128 KB a piece (33 MB of 256 pieces: 8.5 us).  A piece of work is 32 rows of a unit (a wave's) and 4 GROUPS channels of each half of
// the lanes; a workgroup's waves take the unit's records in turn, AT_ONCE of them on the way, and are added up through LDS.
template <bool CAUSAL, int GROUPS, int AT_ONCE>
__global__ __launch_bounds__(64 * TEAMS) void attn_fp8_merge_tiles_kernel(AttnFp8Args a, Layout L)
{
    constexpr int BLOCKS = 16 / GROUPS;
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    const BatchView& b = a.b;
    __shared__ f32x4 part[TEAMS][GROUPS][64];
    __shared__ f32x2 part_ml[TEAMS][64];
    const int lane = threadIdx.x & 63, team = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Plan plan(b, L);
    if (plan.parts < 2) return;
    for (int work = blockIdx.x; work < plan.rest * (NW * BLOCKS); work += gridDim.x) {
        const Unit u = plan.unit(plan.full + work / (NW * BLOCKS));
        const Extent e = extent_of<CAUSAL>(b, L, u, L.units_max <= PLACES);
        const int wave = work / BLOCKS % NW, block = work % BLOCKS;
        const int row = e.row0 + 32 * wave + (lane & 31);
        if (e.pieces < 2 || e.row0 + 32 * wave >= e.n_rows) continue;
        const float* rec = (const float*)a.workspace + (long long)(u.slot * u.parts) * RECORD_FLOATS;
        const int col = 64 * wave + lane;
        f32x4 acc[GROUPS] = {};
        float top = -INFINITY, sum = 0.f;
        auto raise = [&](float to) -> float {                // what there is in terms of a larger reference
            const float ref = to == -INFINITY ? 0.f : to, f = __builtin_amdgcn_exp2f(top - ref);
            top = to;
            sum *= f;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) acc[g] *= f;
            return ref;
        };
        auto take = [&](const f32x4 (&x)[GROUPS], f32x2 ml, float ref) {
            const float f = __builtin_amdgcn_exp2f(ml[0] - ref);
            sum = fmaf(ml[1], f, sum);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[g][k] = fmaf(x[g][k], f, acc[g][k]);
        };
        for (int from = team; from < e.pieces; from += TEAMS * AT_ONCE) {
            f32x4 x[AT_ONCE][GROUPS];
            f32x2 ml[AT_ONCE];
#pragma unroll
            for (int p = 0; p < AT_ONCE; ++p) {
                if (p > 0 && from + TEAMS * p >= e.pieces) break;
                const float* one = rec + (long long)(from + TEAMS * p) * RECORD_FLOATS;
                ml[p] = *(const f32x2*)(one + 64 * 64 * NW + 2 * col);
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) x[p][g] = *(const f32x4*)(one + ((GROUPS * block + g) * 64 * NW + col) * 4);
            }
            float most = top;
#pragma unroll
            for (int p = 0; p < AT_ONCE; ++p)
                if (from + TEAMS * p < e.pieces) most = fmaxf(most, ml[p][0]);
            const float ref = raise(most);
#pragma unroll
            for (int p = 0; p < AT_ONCE; ++p)
                if (from + TEAMS * p < e.pieces) take(x[p], ml[p], ref);
        }
        __syncthreads();                                     // the last piece of work's sums have been read
        if (team > 0) {
            part_ml[team][lane] = f32x2{top, sum};
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) part[team][g][lane] = acc[g];
        }
        __syncthreads();
        if (team > 0) continue;
        float most = top;
#pragma unroll
        for (int w = 1; w < TEAMS; ++w) most = fmaxf(most, part_ml[w][lane][0]);
        const float ref = raise(most);
#pragma unroll
        for (int w = 1; w < TEAMS; ++w) {
            f32x4 x[GROUPS];
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) x[g] = part[w][g][lane];
            take(x, part_ml[w][lane], ref);
        }
        if (row < e.n_rows) {
            const int t = L.by_G.quotient(row);
            const long long place = (long long)(e.first_row + t) * b.num_q_heads + u.kvh * L.G + row - t * L.G;
            const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                bf16x4 w;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = (__bf16)(acc[g][k] * inv);
                *(bf16x4*)((__bf16*)a.out + place * HEAD_DIM + 8 * (GROUPS * block + g) + 4 * (lane >> 5)) = w;
            }
            if (a.lse != nullptr && block == 0 && lane < 32) a.lse[place] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
        }
    }
}

Layout layout_of(const BatchView& b)
{
    Layout L;
    L.G = b.num_q_heads / b.num_kv_heads;
    L.by_G = divisor_of(L.G);
    L.by_kv_heads = divisor_of(b.num_kv_heads);
    const long long longest = ((long long)b.max_new_len * L.G + BR - 1) / BR;
    const long long most = (long long)b.total_new_tokens * L.G / BR + b.num_reqs;
    const bool equal = (long long)b.max_new_len * b.num_reqs == b.total_new_tokens;
    const long long row_tiles = equal ? longest * b.num_reqs : longest * b.num_reqs < most ? longest * b.num_reqs : most;
    const long long units = row_tiles * b.num_kv_heads;
    L.units_max = (int)((units + 7) / 8 * 8);
    // behind whole rounds only long pieces pay; where all units run at once any do
    const long long tiles = ((long long)b.max_pages * b.page_size + BC - 1) / BC;
    L.cut = tiles >= 2 * (L.units_max <= PLACES ? MIN_TILES_ALONE : MIN_TILES_BEHIND) && !(equal && (units + 7) / 8 * 8 % PLACES > PLACES / 2);
    return L;
}

template <bool CAUSAL, int GROUPS, int AT_ONCE>
void merge(const AttnFp8Args& a, const Layout& L, hipStream_t stream)
{
    const int most = std::min(L.units_max, PLACES / 2) * (NW * 16 / GROUPS);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(attn_fp8_merge_tiles_kernel<CAUSAL, GROUPS, AT_ONCE>), dim3(std::min(most, MERGERS)), dim3(64 * TEAMS), 0, stream, a, L);
}

}  // namespace

size_t attn_fp8_tiles_workspace_bytes(const BatchView& b)
{
    return layout_of(b).cut ? (size_t)PLACES * RECORD_FLOATS * sizeof(float) : 0;
}

hipError_t launch_attn_fp8_tiles(const AttnFp8Args& a, bool causal, hipStream_t stream)
{
    const Layout L = layout_of(a.b);
    const dim3 grid((unsigned)(L.units_max + (L.cut ? PLACES : 0))), block(64 * NW);
    if (causal) hipLaunchKernelGGL(attn_fp8_tiles_kernel<true>, grid, block, 0, stream, a, L);
    else hipLaunchKernelGGL(attn_fp8_tiles_kernel<false>, grid, block, 0, stream, a, L);
    if (L.cut) {
        // 32 channels at a time, or 16 with twice the records on the way where few units would leave compute units without work (8 tokens
        // behind 16 k: 17.9 and 19.5 us; 8 images' chunks 65.2 and 64.6, 16 short ones 52.8 and 49.4)
        if (L.units_max <= FEW_UNITS) causal ? merge<true, 2, 8>(a, L, stream) : merge<false, 2, 8>(a, L, stream);
        else causal ? merge<true, 4, 4>(a, L, stream) : merge<false, 4, 4>(a, L, stream);
    }
    return hipGetLastError();
}

}  // namespace emm
