// Entry points of rotary positions (include/emm.h) and of the 8-bit cache (include/emm_fp8.h): validation and dispatch.
// All checks that can fail run before the first HIP call.
#include "../../include/emm_fp8.h"
#include "api_checks.h"
#include "fp8_internal.h"

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>

using emm::MOST_SLOTS;
using emm::api::aligned16;
using emm::api::check_arrays;
using emm::api::check_scalars;
using emm::api::page_size_ok;
using emm::api::view_of;

namespace {

constexpr int64_t MOST_TOKENS = int64_t(1) << 25, MOST_HEADS = 4096, MOST_ROWS = int64_t(1) << 30, MOST_PAIRS = int64_t(1) << 20;

// what the row kernels take: pages as everywhere, both dtypes, heads of 64 or 128, and numbers that their grids and indexes hold
emm_status check_rows(const emm_batch* b)
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

emm_status check_rope(const emm_batch* b, const emm_rope_params* r)
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

emm_status check_rope_arrays(const emm_rope_params* r)
{
    if (r->inv_freq == nullptr || (r->num_axes > 0 && r->positions == nullptr)) return EMM_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(r->inv_freq) & 7u) != 0 || (reinterpret_cast<uintptr_t>(r->positions) & 3u) != 0) return EMM_ERR_INVALID_ARG;
    return EMM_OK;
}

emm::RopeView view_of(const emm_rope_params* r)
{
    emm::RopeView v = {};
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

int64_t elt_bytes(const emm_batch* b) { return b->dtype == EMM_BF16 ? 2 : 4; }

// elements between rows of `heads` heads, given what the caller says about them; -1: refused
int64_t stride_of(const emm_batch* b, int64_t heads, int64_t token_stride)
{
    const int64_t row = heads * b->head_dim;
    if (token_stride == 0) return row;
    // (rows that span 2^60 bytes are in no memory, and what follows counts them in 64 bits)
    if (token_stride < row || token_stride > (int64_t(1) << 60) / elt_bytes(b) / std::max(b->total_new_tokens, 1)) return -1;
    if (token_stride * elt_bytes(b) % 16 != 0) return -1;
    return token_stride;
}

// do rows that are read through a stride and packed rows that are written share memory?
bool overlap(const emm_batch* b, const void* in, int64_t in_stride, int64_t in_heads, const void* out, int64_t out_heads)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(in), y = reinterpret_cast<uintptr_t>(out);
    const uintptr_t x_end = x + static_cast<uintptr_t>(((b->total_new_tokens - 1) * in_stride + in_heads * b->head_dim) * elt_bytes(b));
    const uintptr_t y_end = y + static_cast<uintptr_t>(b->total_new_tokens * out_heads * b->head_dim * elt_bytes(b));
    return x < y_end && y < x_end;
}
// a tensor's own output: in place (each value is read before it is written) or apart from it
bool own_output_ok(const emm_batch* b, const void* in, int64_t in_stride, int64_t heads, const void* out)
{
    return (in == out && in_stride == heads * b->head_dim) || !overlap(b, in, in_stride, heads, out, heads);
}

emm_status check_cache(const emm_batch* b, const emm_fp8_cache* c)
{
    if (c == nullptr || c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr) return EMM_ERR_NULL;
    for (const void* p : {c->k, c->v, c->k_scale, c->v_scale})
        if (!aligned16(p)) return EMM_ERR_INVALID_ARG;
    if (b->num_pages == 0 || b->max_pages_per_req == 0) return EMM_ERR_INVALID_ARG;
    return EMM_OK;
}

emm::Fp8Pools pools_of(const emm_fp8_cache* c)
{
    return emm::Fp8Pools{static_cast<unsigned char*>(c->k), static_cast<unsigned char*>(c->v), static_cast<unsigned char*>(c->k_scale),
                         static_cast<unsigned char*>(c->v_scale)};
}

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
