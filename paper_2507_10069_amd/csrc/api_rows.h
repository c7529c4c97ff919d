// Host-side checks that the entry points of rows share: rotary positions, norms, the 8-bit cache (include/emm.h, emm_fp8.h, emm_step.h).
#pragma once

#include "../../include/emm_fp8.h"
#include "api_checks.h"
#include "fp8_internal.h"

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>

namespace emm {
namespace api {

constexpr int64_t MOST_TOKENS = int64_t(1) << 25, MOST_HEADS = 4096, MOST_ROWS = int64_t(1) << 30, MOST_PAIRS = int64_t(1) << 20;

// what the row kernels take: pages as everywhere, both dtypes, heads of 64 or 128, and numbers that their grids and indexes hold
inline emm_status check_rows(const emm_batch* b)
{
    const emm_status st = check_scalars(b);
    if (st != EMM_OK) return st;
    if (!page_size_ok(b)) return EMM_ERR_UNSUPPORTED;
    if (b->head_dim != 64 && b->head_dim != 128) return EMM_ERR_UNSUPPORTED;
    if (b->total_new_tokens > MOST_TOKENS || b->num_q_heads > MOST_HEADS || int64_t(b->total_new_tokens) * b->num_q_heads > MOST_ROWS ||
        int64_t(b->max_pages_per_req) * b->page_size > MOST_SLOTS)
        return EMM_ERR_UNSUPPORTED;
    return EMM_OK;
}

inline emm_status check_rope(const emm_batch* b, const emm_rope_params* r)
{
    if (r == nullptr) return EMM_ERR_NULL;
    if (r->layout != EMM_ROPE_HALF && r->layout != EMM_ROPE_INTERLEAVED) return EMM_ERR_INVALID_ARG;
    if (r->rotary_dim <= 0 || r->rotary_dim > b->head_dim) return EMM_ERR_INVALID_ARG;
    if (r->rotary_dim % 16 != 0) return EMM_ERR_UNSUPPORTED;
    if (r->num_axes < 0 || r->num_axes > 4 || (r->inverse != 0 && r->inverse != 1) || r->reserved != 0 || !std::isfinite(r->factor))
        return EMM_ERR_INVALID_ARG;
    int64_t sum = 0;
    for (int a = 0; a < r->num_axes; ++a) {
        if (r->sections[a] < 0) return EMM_ERR_INVALID_ARG;
        sum += r->sections[a];
    }
    if (r->num_axes > 0 && sum != r->rotary_dim / 2) return EMM_ERR_INVALID_ARG;
    if (r->num_axes == 0 && r->positions != nullptr) return EMM_ERR_INVALID_ARG;
    return EMM_OK;
}

inline emm_status check_rope_arrays(const emm_rope_params* r)
{
    if (r->inv_freq == nullptr || (r->num_axes > 0 && r->positions == nullptr)) return EMM_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(r->inv_freq) & 7u) != 0 || (reinterpret_cast<uintptr_t>(r->positions) & 3u) != 0) return EMM_ERR_INVALID_ARG;
    return EMM_OK;
}

inline RopeView view_of(const emm_rope_params* r)
{
    RopeView v = {};
    v.inv_freq = r->inv_freq;
    v.positions = r->num_axes > 0 ? r->positions : nullptr;
    v.rotary_dim = r->rotary_dim;
    v.interleaved = r->layout == EMM_ROPE_INTERLEAVED;
    v.num_axes = r->num_axes;
    int sum = 0;
    for (int a = 0; a < 3; ++a) {
        sum += a < r->num_axes ? r->sections[a] : r->rotary_dim;
        v.ends[a] = sum;
    }
    v.factor = r->factor;
    v.sine_factor = r->inverse ? -r->factor : r->factor;
    return v;
}

inline int64_t elt_bytes(const emm_batch* b) { return b->dtype == EMM_BF16 ? 2 : 4; }

// elements between rows of `heads` heads, given what the caller says about them; -1: refused
inline int64_t stride_of(const emm_batch* b, int64_t heads, int64_t token_stride)
{
    const int64_t row = heads * b->head_dim;
    if (token_stride == 0) return row;
    // (rows that span 2^60 bytes are in no memory, and what follows counts them in 64 bits)
    if (token_stride < row || token_stride > (int64_t(1) << 60) / elt_bytes(b) / std::max(b->total_new_tokens, 1)) return -1;
    if (token_stride * elt_bytes(b) % 16 != 0) return -1;
    return token_stride;
}

// do rows that are read through a stride and packed rows that are written share memory?
inline bool overlap(const emm_batch* b, const void* in, int64_t in_stride, int64_t in_heads, const void* out, int64_t out_heads)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(in), y = reinterpret_cast<uintptr_t>(out);
    const uintptr_t x_end = x + static_cast<uintptr_t>(((b->total_new_tokens - 1) * in_stride + in_heads * b->head_dim) * elt_bytes(b));
    const uintptr_t y_end = y + static_cast<uintptr_t>(b->total_new_tokens * out_heads * b->head_dim * elt_bytes(b));
    return x < y_end && y < x_end;
}
// a tensor's own output: in place (each value is read before it is written) or apart from it
inline bool own_output_ok(const emm_batch* b, const void* in, int64_t in_stride, int64_t heads, const void* out)
{
    return (in == out && in_stride == heads * b->head_dim) || !overlap(b, in, in_stride, heads, out, heads);
}

inline emm_status check_cache(const emm_batch* b, const emm_fp8_cache* c)
{
    if (c == nullptr || c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr) return EMM_ERR_NULL;
    for (const void* p : {c->k, c->v, c->k_scale, c->v_scale})
        if (!aligned16(p)) return EMM_ERR_INVALID_ARG;
    if (b->num_pages == 0 || b->max_pages_per_req == 0) return EMM_ERR_INVALID_ARG;
    return EMM_OK;
}

inline Fp8Pools pools_of(const emm_fp8_cache* c)
{
    return Fp8Pools{static_cast<unsigned char*>(c->k), static_cast<unsigned char*>(c->v), static_cast<unsigned char*>(c->k_scale),
                         static_cast<unsigned char*>(c->v_scale)};
}

}  // namespace api
}  // namespace emm
