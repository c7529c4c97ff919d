// Host-side checks that every entry point of the library makes, and the device view of a batch.
#pragma once

#include "../../include/emm.h"
#include "emm_internal.h"

#include <cmath>
#include <cstdint>

namespace emm {
namespace api {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline emm_status check_scalars(const emm_batch* b)
{
    if (b == nullptr) return EMM_ERR_NULL;
    if (b->num_reqs < 0 || b->num_q_heads <= 0 || b->num_kv_heads <= 0 || b->head_dim <= 0 ||
        b->page_size <= 0 || b->num_pages < 0 || b->max_pages_per_req < 0 || b->total_new_tokens < 0 ||
        b->max_new_len < 0 || b->max_new_len > b->total_new_tokens || b->reserved != 0)
        return EMM_ERR_INVALID_ARG;
    if (b->num_q_heads % b->num_kv_heads != 0) return EMM_ERR_INVALID_ARG;
    if (b->dtype != EMM_F32 && b->dtype != EMM_BF16) return EMM_ERR_INVALID_ARG;
    if (!(b->softmax_scale > 0.0f) || !std::isfinite(b->softmax_scale)) return EMM_ERR_INVALID_ARG;
    if (b->num_reqs > 0 && b->total_new_tokens > 0 && b->max_new_len == 0) return EMM_ERR_INVALID_ARG;
    return EMM_OK;
}

inline bool page_size_ok(const emm_batch* b)
{
    return b->page_size == 16 || b->page_size == 32 || b->page_size == 64 || b->page_size == 128 || b->page_size == 256;
}

inline emm_status check_arrays(const emm_batch* b)
{
    if (b->num_reqs == 0) return EMM_OK;
    if (b->page_table == nullptr || b->prefix_lens == nullptr || b->new_lens == nullptr ||
        b->cu_new_lens == nullptr)
        return EMM_ERR_NULL;
    return EMM_OK;
}

inline BatchView view_of(const emm_batch* b)
{
    BatchView v;
    v.page_table = b->page_table;
    v.prefix_lens = b->prefix_lens;
    v.new_lens = b->new_lens;
    v.cu_new_lens = b->cu_new_lens;
    v.num_reqs = b->num_reqs;
    v.num_q_heads = b->num_q_heads;
    v.num_kv_heads = b->num_kv_heads;
    v.head_dim = b->head_dim;
    v.page_size = b->page_size;
    v.page_shift = 0;
    while ((16 << v.page_shift) < b->page_size) ++v.page_shift;
    v.num_pages = b->num_pages;
    v.max_pages = b->max_pages_per_req;
    v.total_new_tokens = b->total_new_tokens;
    v.max_new_len = b->max_new_len;
    v.softmax_scale = b->softmax_scale;
    return v;
}

}  // namespace api
}  // namespace emm
