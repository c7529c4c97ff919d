// Entry points of rotary positions (include/emm.h) and of the 8-bit cache (include/emm_fp8.h): validation and dispatch.
// All checks that can fail run before the first HIP call.
#include "api_rows.h"

using namespace emm::api;

namespace {

// k_new and v_new (and, with a rotation, q) into the cache
emm_status scatter(const emm_batch* b, const emm_rope_params* rope, const void* q, const void* k_new, const void* v_new, int64_t token_stride,
                   void* q_out, const emm_fp8_cache* cache, void* hip_stream)
{
    emm_status st = check_rows(b);
    if (st != EMM_OK) return st;
    if (rope != nullptr && (st = check_rope(b, rope)) != EMM_OK) return st;
    const int64_t sq = rope != nullptr ? stride_of(b, b->num_q_heads, token_stride) : 0, skv = stride_of(b, b->num_kv_heads, token_stride);
    if (sq < 0 || skv < 0) return EMM_ERR_INVALID_ARG;
    if (b->total_new_tokens == 0) return EMM_OK;
    // (without requests nothing is written, but given positions turn q's rows all the same)
    if (b->num_reqs == 0) return rope != nullptr && rope->num_axes > 0 ? emm_rope(b, rope, q, nullptr, token_stride, q_out, nullptr, hip_stream) : EMM_OK;
    if ((st = check_arrays(b)) != EMM_OK) return st;
    if (rope != nullptr && (st = check_rope_arrays(rope)) != EMM_OK) return st;
    if (k_new == nullptr || v_new == nullptr || (rope != nullptr && (q == nullptr || q_out == nullptr))) return EMM_ERR_NULL;
    if ((st = check_cache(b, cache)) != EMM_OK) return st;
    if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(q) || !aligned16(q_out)) return EMM_ERR_INVALID_ARG;
    if (rope != nullptr && (!own_output_ok(b, q, sq, b->num_q_heads, q_out) || overlap(b, k_new, skv, b->num_kv_heads, q_out, b->num_q_heads) ||
                            overlap(b, v_new, skv, b->num_kv_heads, q_out, b->num_q_heads)))
        return EMM_ERR_INVALID_ARG;
    const emm::NewRows rows = {q, k_new, v_new, sq, skv, skv, q_out, nullptr};
    const emm::Fp8Pools pools = pools_of(cache);
    const hipError_t err = emm::launch_rope_rows(view_of(b), b->dtype == EMM_BF16, rope != nullptr ? view_of(rope) : emm::RopeView{}, rows, &pools,
                                                 static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? EMM_OK : EMM_ERR_LAUNCH;
}

emm_status attention(const emm_batch* b, const void* q, const emm_fp8_cache* cache, void* out, float* lse, void* workspace, size_t workspace_bytes,
                     void* hip_stream, bool causal)
{
    size_t need = 0;
    emm_status st = emm_attn_fp8_workspace_size(b, &need);
    if (st != EMM_OK) return st;
    if (b->num_reqs == 0 || b->total_new_tokens == 0) return EMM_OK;
    if ((st = check_arrays(b)) != EMM_OK) return st;
    if (q == nullptr || out == nullptr) return EMM_ERR_NULL;
    if ((st = check_cache(b, cache)) != EMM_OK) return st;
    if (need > 0 && workspace == nullptr) return EMM_ERR_NULL;
    if (workspace_bytes < need) return EMM_ERR_WORKSPACE;
    if (!aligned16(q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(lse) & 3u) != 0 || !aligned16(workspace)) return EMM_ERR_INVALID_ARG;
    const emm::AttnFp8Args args = {view_of(b), q, pools_of(cache), out, lse, need > 0 ? workspace : nullptr};
    const hipError_t err = emm::launch_attn_fp8(args, causal, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? EMM_OK : EMM_ERR_LAUNCH;
}

}  // namespace

extern "C" {

emm_status emm_rope_inv_freq_host(const emm_rope_scaling* s, double* inv_freq, float* factor)
{
    if (s == nullptr || inv_freq == nullptr) return EMM_ERR_NULL;
    if (s->rotary_dim < 16 || s->rotary_dim > 128 || s->rotary_dim % 16 != 0 || s->reserved != 0 || s->kind < EMM_ROPE_PLAIN || s->kind > EMM_ROPE_BANDS)
        return EMM_ERR_INVALID_ARG;
    if (!(s->base > 1.0) || !std::isfinite(s->base) || !(s->scale >= 1.0) || !std::isfinite(s->scale)) return EMM_ERR_INVALID_ARG;
    const bool ramp = s->kind == EMM_ROPE_YARN || s->kind == EMM_ROPE_BANDS;
    if (ramp && (s->original_len <= 0 || !(s->slow > 0.0) || !(s->fast > s->slow) || !std::isfinite(s->fast))) return EMM_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925286766559, n = s->rotary_dim;
    const double base = s->kind == EMM_ROPE_NTK ? s->base * std::pow(s->scale, n / (n - 2.0)) : s->base;
    // the (fractional) frequency that makes `turns` turns in original_len tokens
    auto index_of = [&](double turns) { return n * std::log(s->original_len / (turns * two_pi)) / (2.0 * std::log(s->base)); };
    const double lo = ramp ? std::max(std::floor(index_of(s->fast)), 0.0) : 0.0;
    const double hi = ramp ? std::max(std::min(std::ceil(index_of(s->slow)), n - 1.0), lo + 0.001) : 1.0;
    // (the ramp's ends are held at frequency 0 or above; where even that one turns less than `slow` times there is no ramp)
    const bool none_kept = s->kind == EMM_ROPE_LINEAR || (ramp && index_of(s->slow) < 0.0);
    for (int i = 0; i < s->rotary_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / n);
        double kept = none_kept ? 0.0 : 1.0;                 // share of the frequency that is not divided by scale
        if (s->kind == EMM_ROPE_YARN && !none_kept) kept = 1.0 - std::min(std::max((i - lo) / (hi - lo), 0.0), 1.0);
        if (s->kind == EMM_ROPE_BANDS && !none_kept) kept = std::min(std::max((s->original_len * f / two_pi - s->slow) / (s->fast - s->slow), 0.0), 1.0);
        inv_freq[i] = f * kept + f / s->scale * (1.0 - kept);
    }
    if (factor != nullptr) *factor = s->kind == EMM_ROPE_YARN ? static_cast<float>(0.1 * std::log(s->scale) + 1.0) : 1.0f;
    return EMM_OK;
}

emm_status emm_rope(const emm_batch* b, const emm_rope_params* rope, const void* q, const void* k, int64_t token_stride, void* q_out, void* k_out,
                    void* hip_stream)
{
    emm_status st = check_rows(b);
    if (st != EMM_OK) return st;
    if ((st = check_rope(b, rope)) != EMM_OK) return st;
    // (a pair that is not given has no row that the stride must hold)
    const int64_t sq = q != nullptr ? stride_of(b, b->num_q_heads, token_stride) : 0, sk = k != nullptr ? stride_of(b, b->num_kv_heads, token_stride) : 0;
    if (sq < 0 || sk < 0) return EMM_ERR_INVALID_ARG;
    // (given positions belong to rows, whether or not a request has them)
    if (b->total_new_tokens == 0 || (b->num_reqs == 0 && rope->num_axes == 0)) return EMM_OK;
    if (rope->num_axes == 0 && (st = check_arrays(b)) != EMM_OK) return st;
    if ((st = check_rope_arrays(rope)) != EMM_OK) return st;
    if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr) || (q == nullptr && k == nullptr)) return EMM_ERR_NULL;
    for (const void* p : {q, k, static_cast<const void*>(q_out), static_cast<const void*>(k_out)})
        if (!aligned16(p)) return EMM_ERR_INVALID_ARG;
    const int64_t hq = b->num_q_heads, hk = b->num_kv_heads;
    if ((q != nullptr && !own_output_ok(b, q, sq, hq, q_out)) || (k != nullptr && !own_output_ok(b, k, sk, hk, k_out))) return EMM_ERR_INVALID_ARG;
    if (q != nullptr && k != nullptr &&
        (overlap(b, q, sq, hq, k_out, hk) || overlap(b, k, sk, hk, q_out, hq) || overlap(b, q_out, hq * b->head_dim, hq, k_out, hk)))
        return EMM_ERR_INVALID_ARG;
    const emm::NewRows rows = {q, k, nullptr, sq, sk, 0, q_out, k_out};
    const hipError_t err = emm::launch_rope_rows(view_of(b), b->dtype == EMM_BF16, view_of(rope), rows, nullptr, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? EMM_OK : EMM_ERR_LAUNCH;
}

emm_status emm_kv_scatter_fp8(const emm_batch* b, const void* k_new, const void* v_new, int64_t token_stride, const emm_fp8_cache* cache,
                              void* hip_stream)
{
    return scatter(b, nullptr, nullptr, k_new, v_new, token_stride, nullptr, cache, hip_stream);
}

emm_status emm_rope_kv_scatter_fp8(const emm_batch* b, const emm_rope_params* rope, const void* q, const void* k_new, const void* v_new,
                                   int64_t token_stride, void* q_out, const emm_fp8_cache* cache, void* hip_stream)
{
    if (b != nullptr && rope == nullptr) return EMM_ERR_NULL;
    return scatter(b, rope, q, k_new, v_new, token_stride, q_out, cache, hip_stream);
}

emm_status emm_kv_gather_fp8(const emm_batch* b, const emm_fp8_cache* cache, void* k_out, void* v_out, void* hip_stream)
{
    emm_status st = check_rows(b);
    if (st != EMM_OK) return st;
    if (b->num_reqs == 0 || b->total_new_tokens == 0) return EMM_OK;
    if ((st = check_arrays(b)) != EMM_OK) return st;
    if (k_out == nullptr || v_out == nullptr) return EMM_ERR_NULL;
    if ((st = check_cache(b, cache)) != EMM_OK) return st;
    if (!aligned16(k_out) || !aligned16(v_out)) return EMM_ERR_INVALID_ARG;
    const hipError_t err = emm::launch_kv_gather_fp8(view_of(b), b->dtype == EMM_BF16, pools_of(cache), k_out, v_out, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? EMM_OK : EMM_ERR_LAUNCH;
}

emm_status emm_attn_fp8_workspace_size(const emm_batch* b, size_t* bytes)
{
    if (bytes == nullptr) return EMM_ERR_NULL;
    *bytes = 0;
    const emm_status st = check_rows(b);
    if (st != EMM_OK) return st;
    if (b->dtype != EMM_BF16 || b->head_dim != 128 || int64_t(b->num_reqs) * b->num_kv_heads > MOST_PAIRS) return EMM_ERR_UNSUPPORTED;
    *bytes = emm::attn_fp8_workspace_bytes(view_of(b));
    return EMM_OK;
}

emm_status emm_prefill_attn_fp8(const emm_batch* b, const void* q, const emm_fp8_cache* cache, void* out, float* lse, void* workspace,
                                size_t workspace_bytes, void* hip_stream)
{
    return attention(b, q, cache, out, lse, workspace, workspace_bytes, hip_stream, true);
}

emm_status emm_cross_attn_fp8(const emm_batch* b, const void* q, const emm_fp8_cache* cache, void* out, float* lse, void* workspace,
                              size_t workspace_bytes, void* hip_stream)
{
    return attention(b, q, cache, out, lse, workspace, workspace_bytes, hip_stream, false);
}

emm_status emm_decode_attn_fp8(const emm_batch* b, const void* q, const emm_fp8_cache* cache, void* out, float* lse, void* workspace,
                               size_t workspace_bytes, void* hip_stream)
{
    if (b != nullptr && b->max_new_len > 1) return EMM_ERR_INVALID_ARG;
    return attention(b, q, cache, out, lse, workspace, workspace_bytes, hip_stream, true);
}

}  // extern "C"
