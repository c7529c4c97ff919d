// Entry points of include/emm_step.h: validation and dispatch.  All checks that can fail run before the first HIP call.
#include "../../include/emm_step.h"
#include "api_rows.h"
#include "step_internal.h"

#include <cfloat>

using namespace emm::api;

namespace {

emm_status check_norm(const emm_qk_norm* n)
{
    if (n->reserved != 0 || !(n->eps >= FLT_MIN) || !std::isfinite(n->eps)) return EMM_ERR_INVALID_ARG;
    return EMM_OK;
}

// A row call's tensors as the checks see them.  cached: k and v go into a cache, else k into k_out
struct RowCall {
    const emm_qk_norm* norm;
    const emm_rope_params* rope;
    const void *q, *k, *v;
    int64_t token_stride;
    const int64_t* slots;
    void *q_out, *k_out;
    bool cached;
    const emm_fp8_cache* fp8;
    void *k_cache, *v_cache;
};

bool from_batch(const RowCall& c) { return c.rope != nullptr && c.rope->num_axes == 0; }

emm_status rows(const emm_batch* b, RowCall c, void* hip_stream)
{
    emm_status st = check_rows(b);
    if (st != EMM_OK) return st;
    if (c.norm == nullptr && c.rope == nullptr) return EMM_ERR_NULL;
    if (c.norm != nullptr && (st = check_norm(c.norm)) != EMM_OK) return st;
    if (c.rope != nullptr && (st = check_rope(b, c.rope)) != EMM_OK) return st;
    const int64_t hq = b->num_q_heads, hk = b->num_kv_heads;
    const bool with_q = c.cached || c.q != nullptr, with_k = c.cached || c.k != nullptr;     // (a tensor that is not given has no row that the stride must hold)
    const int64_t sq = with_q ? stride_of(b, hq, c.token_stride) : 0, sk = with_k ? stride_of(b, hk, c.token_stride) : 0;
    if (sq < 0 || sk < 0) return EMM_ERR_INVALID_ARG;
    if (b->total_new_tokens == 0 || (b->num_reqs == 0 && from_batch(c))) return EMM_OK;
    if ((from_batch(c) || (c.cached && c.slots == nullptr)) && (st = check_arrays(b)) != EMM_OK) return st;
    if (c.rope != nullptr && (st = check_rope_arrays(c.rope)) != EMM_OK) return st;
    if (c.norm != nullptr && (c.norm->q_weight == nullptr || c.norm->k_weight == nullptr)) return EMM_ERR_NULL;
    if (c.norm != nullptr && (!aligned16(c.norm->q_weight) || !aligned16(c.norm->k_weight))) return EMM_ERR_INVALID_ARG;
    if (c.cached) {
        if (c.q == nullptr || c.q_out == nullptr || c.k == nullptr || c.v == nullptr) return EMM_ERR_NULL;
    } else if ((c.q == nullptr) != (c.q_out == nullptr) || (c.k == nullptr) != (c.k_out == nullptr) || (c.q == nullptr && c.k == nullptr)) {
        return EMM_ERR_NULL;
    }
    for (const void* p : {c.q, c.k, c.v, static_cast<const void*>(c.q_out), static_cast<const void*>(c.k_out)})
        if (!aligned16(p)) return EMM_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(c.slots) & 7u) != 0) return EMM_ERR_INVALID_ARG;
    if (c.q != nullptr && !own_output_ok(b, c.q, sq, hq, c.q_out)) return EMM_ERR_INVALID_ARG;
    if (c.cached) {
        if (overlap(b, c.k, sk, hk, c.q_out, hq) || overlap(b, c.v, sk, hk, c.q_out, hq)) return EMM_ERR_INVALID_ARG;
        // (given slots are of the pools alone; those of the batch want a table)
        if (b->num_pages == 0 || (c.slots == nullptr && b->num_reqs > 0 && b->max_pages_per_req == 0)) return EMM_ERR_INVALID_ARG;
        if (c.fp8 != nullptr) {
            emm_batch pools = *b;
            pools.max_pages_per_req = 1;
            if ((st = check_cache(&pools, c.fp8)) != EMM_OK) return st;
        } else {
            if (c.k_cache == nullptr || c.v_cache == nullptr) return EMM_ERR_NULL;
            if (!aligned16(c.k_cache) || !aligned16(c.v_cache)) return EMM_ERR_INVALID_ARG;
        }
    } else {
        if (c.k != nullptr && !own_output_ok(b, c.k, sk, hk, c.k_out)) return EMM_ERR_INVALID_ARG;
        if (c.q != nullptr && c.k != nullptr &&
            (overlap(b, c.q, sq, hq, c.k_out, hk) || overlap(b, c.k, sk, hk, c.q_out, hq) || overlap(b, c.q_out, hq * b->head_dim, hq, c.k_out, hk)))
            return EMM_ERR_INVALID_ARG;
    }
    bool cached = c.cached;
    if (cached && c.slots == nullptr && b->num_reqs == 0) {  // no row has a slot: q alone
        cached = false;
        c.k = c.v = nullptr;
    }
    emm::NormView norm = {nullptr, nullptr, 0.0f, c.slots};
    if (c.norm != nullptr) norm = {c.norm->q_weight, c.norm->k_weight, c.norm->eps, c.slots};
    const emm::NewRows rows = {c.q, c.k, c.v, sq, sk, sk, c.q_out, c.k_out};
    const emm::Fp8Pools fp8 = c.fp8 != nullptr ? pools_of(c.fp8) : emm::Fp8Pools{};
    const emm::PlainPools plain = {c.k_cache, c.v_cache};
    const hipError_t err = emm::launch_norm_rope_rows(view_of(b), b->dtype == EMM_BF16, norm, c.rope != nullptr ? view_of(c.rope) : emm::RopeView{}, rows,
                                                      cached && c.fp8 != nullptr ? &fp8 : nullptr, cached && c.fp8 == nullptr ? &plain : nullptr,
                                                      static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? EMM_OK : EMM_ERR_LAUNCH;
}

emm_status check_window(const emm_batch* b, int32_t window, int32_t sinks)
{
    const emm_status st = check_rows(b);
    if (st != EMM_OK) return st;
    if (window < 1 || sinks < 0) return EMM_ERR_INVALID_ARG;
    if (b->dtype == EMM_BF16 && b->head_dim != 128) return EMM_ERR_UNSUPPORTED;
    if (int64_t(b->num_reqs) * b->num_kv_heads > MOST_PAIRS) return EMM_ERR_UNSUPPORTED;
    return EMM_OK;
}

emm_status attention(const emm_batch* b, int32_t window, int32_t sinks, const void* q, const void* k_cache, const void* v_cache, void* out, float* lse,
                     void* workspace, size_t workspace_bytes, void* hip_stream)
{
    size_t need = 0;
    emm_status st = emm_attn_window_workspace_size(b, window, sinks, &need);
    if (st != EMM_OK) return st;
    if (b->num_reqs == 0 || b->total_new_tokens == 0) return EMM_OK;
    if ((st = check_arrays(b)) != EMM_OK) return st;
    if (q == nullptr || k_cache == nullptr || v_cache == nullptr || out == nullptr) return EMM_ERR_NULL;
    if (b->num_pages == 0 || b->max_pages_per_req == 0) return EMM_ERR_INVALID_ARG;
    if (need > 0 && workspace == nullptr) return EMM_ERR_NULL;
    if (workspace_bytes < need) return EMM_ERR_WORKSPACE;
    for (const void* p : {q, k_cache, v_cache, static_cast<const void*>(out), static_cast<const void*>(workspace)})
        if (!aligned16(p)) return EMM_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(lse) & 3u) != 0) return EMM_ERR_INVALID_ARG;
    emm::AttnArgs args = {view_of(b), q, k_cache, v_cache, out, lse, 1, need > 0 ? workspace : nullptr};
    const emm::WindowView w = {window, sinks};
    const hipError_t err = b->dtype == EMM_BF16 ? emm::launch_attn_window(args, w, static_cast<hipStream_t>(hip_stream))
                                                : emm::launch_attn_f32_window(args, w, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? EMM_OK : EMM_ERR_LAUNCH;
}

struct Range {
    const void* at;
    int64_t bytes;
};
bool meet(const Range& x, const Range& y)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.at), c = reinterpret_cast<uintptr_t>(y.at);
    return x.at != nullptr && y.at != nullptr && x.bytes > 0 && y.bytes > 0 && a < c + static_cast<uintptr_t>(y.bytes) && c < a + static_cast<uintptr_t>(x.bytes);
}

}  // namespace

extern "C" {

emm_status emm_page_step(const emm_page_step_params* s, void* hip_stream)
{
    if (s == nullptr) return EMM_ERR_NULL;
    if (s->num_reqs < 0 || s->num_pages < 1 || s->max_pages_per_req < 0 || s->max_tokens < 0 || s->window < 0 || s->sinks < 0 || s->reserved != 0)
        return EMM_ERR_INVALID_ARG;
    if (s->num_reqs > 0 && s->max_pages_per_req == 0) return EMM_ERR_INVALID_ARG;
    emm_batch pages = {};
    pages.page_size = s->page_size;
    if (!page_size_ok(&pages) || s->num_reqs > emm::MOST_STEP_REQS || s->num_pages > emm::MOST_STEP_PAGES || s->max_tokens > MOST_TOKENS ||
        int64_t(s->max_pages_per_req) * s->page_size > emm::MOST_SLOTS)
        return EMM_ERR_UNSUPPORTED;
    if (s->free_pages == nullptr || s->free_count == nullptr || s->free_count_out == nullptr || s->cu_new_lens == nullptr) return EMM_ERR_NULL;
    if (s->num_reqs > 0)
        for (const int32_t* p : {static_cast<const int32_t*>(s->page_table), s->lens, s->add_lens, s->held_from, static_cast<const int32_t*>(s->prefix_lens),
                                 static_cast<const int32_t*>(s->new_lens), static_cast<const int32_t*>(s->lens_out), static_cast<const int32_t*>(s->held_out)})
            if (p == nullptr) return EMM_ERR_NULL;
    const int64_t n = 4 * int64_t(s->num_reqs), t = s->max_tokens;
    const Range in[] = {{s->lens, n}, {s->held_from, n}, {s->free_count, 4}, {s->add_lens, n}};
    const Range out[] = {{s->lens_out, n}, {s->held_out, n}, {s->free_count_out, 4}, {s->page_table, n * s->max_pages_per_req}, {s->free_pages, 4 * int64_t(s->num_pages)},
                         {s->prefix_lens, n}, {s->new_lens, n}, {s->cu_new_lens, n + 4}, {s->slots, 8 * t}, {s->positions, 4 * t}, {s->refused, 4}};
    for (const Range& x : in)
        if ((reinterpret_cast<uintptr_t>(x.at) & 3u) != 0) return EMM_ERR_INVALID_ARG;
    for (const Range& x : out)
        if ((reinterpret_cast<uintptr_t>(x.at) & 3u) != 0) return EMM_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(s->slots) & 7u) != 0) return EMM_ERR_INVALID_ARG;
    bool in_place = false;
    for (int o = 0; o < 11; ++o) {
        for (int i = 0; i < 4; ++i) {
            if (o == i && o < 3 && out[o].at == in[i].at) in_place = true;
            else if (meet(out[o], in[i])) return EMM_ERR_INVALID_ARG;
        }
        for (int p = 0; p < o; ++p)
            if (meet(out[o], out[p])) return EMM_ERR_INVALID_ARG;
    }
    int shift = 0;
    while ((16 << shift) < s->page_size) ++shift;
    emm::PageStepArgs a = {};
    a.num_reqs = s->num_reqs;
    a.page_shift = shift;
    a.num_pages = s->num_pages;
    a.max_pages = s->max_pages_per_req;
    a.max_tokens = s->max_tokens;
    a.window = s->window;
    a.sink_pages = static_cast<int32_t>((int64_t(s->sinks) + s->page_size - 1) / s->page_size);
    a.page_table = s->page_table;
    a.free_pages = s->free_pages;
    a.lens = s->lens;
    a.add_lens = s->add_lens;
    a.held_from = s->held_from;
    a.free_count = s->free_count;
    a.prefix_lens = s->prefix_lens;
    a.new_lens = s->new_lens;
    a.cu_new_lens = s->cu_new_lens;
    a.lens_out = s->lens_out;
    a.held_out = s->held_out;
    a.free_count_out = s->free_count_out;
    a.slots = s->slots;
    a.positions = s->positions;
    a.refused = s->refused;
    const hipError_t err = emm::launch_page_step(a, in_place, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? EMM_OK : EMM_ERR_LAUNCH;
}

emm_status emm_norm_rope(const emm_batch* b, const emm_qk_norm* norm, const emm_rope_params* rope, const void* q, const void* k, int64_t token_stride,
                         void* q_out, void* k_out, void* hip_stream)
{
    return rows(b, {norm, rope, q, k, nullptr, token_stride, nullptr, q_out, k_out, false, nullptr, nullptr, nullptr}, hip_stream);
}

emm_status emm_norm_rope_kv_scatter(const emm_batch* b, const emm_qk_norm* norm, const emm_rope_params* rope, const void* q, const void* k_new,
                                    const void* v_new, int64_t token_stride, const int64_t* slots, void* q_out, void* k_cache, void* v_cache, void* hip_stream)
{
    return rows(b, {norm, rope, q, k_new, v_new, token_stride, slots, q_out, nullptr, true, nullptr, k_cache, v_cache}, hip_stream);
}

emm_status emm_norm_rope_kv_scatter_fp8(const emm_batch* b, const emm_qk_norm* norm, const emm_rope_params* rope, const void* q, const void* k_new,
                                        const void* v_new, int64_t token_stride, const int64_t* slots, void* q_out, const emm_fp8_cache* cache,
                                        void* hip_stream)
{
    const emm_fp8_cache none = {};
    return rows(b, {norm, rope, q, k_new, v_new, token_stride, slots, q_out, nullptr, true, cache != nullptr ? cache : &none, nullptr, nullptr}, hip_stream);
}

emm_status emm_attn_window_workspace_size(const emm_batch* b, int32_t window, int32_t sinks, size_t* bytes)
{
    if (bytes == nullptr) return EMM_ERR_NULL;
    *bytes = 0;
    const emm_status st = check_window(b, window, sinks);
    if (st != EMM_OK) return st;
    if (b->dtype == EMM_BF16) *bytes = emm::attn_window_workspace_bytes(view_of(b), emm::WindowView{window, sinks});
    return EMM_OK;
}

emm_status emm_prefill_attn_window(const emm_batch* b, int32_t window, int32_t sinks, const void* q, const void* k_cache, const void* v_cache, void* out,
                                   float* lse, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    return attention(b, window, sinks, q, k_cache, v_cache, out, lse, workspace, workspace_bytes, hip_stream);
}

emm_status emm_decode_attn_window(const emm_batch* b, int32_t window, int32_t sinks, const void* q, const void* k_cache, const void* v_cache, void* out,
                                  float* lse, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (b != nullptr && b->max_new_len > 1) return EMM_ERR_INVALID_ARG;
    return attention(b, window, sinks, q, k_cache, v_cache, out, lse, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
