/*
 * emm_fp8.h -- the KV cache in 8 bits.  The same pools, pages and batches as emm.h, with half of the bytes: a decode
 * step, which is bound by reading K and V, reads half as much, and a pool holds twice the contexts.
 *
 * Format.  A row is the head_dim values of one (token, KV head), of K or of V.  It is held as head_dim codes of
 * 8 bits (OCP E4M3: sign, 4 bits of exponent, 3 of significand, largest 448, no infinities) and one scale byte
 * (E8M0: the power of two 2^(byte - 127)):
 *   most = largest |x| over the row's finite values; e = least integer -117 .. 119 with most <= 448 * 2^e, else 119;
 *   byte = e + 127 (10 .. 246); code = x * 2^-e rounded to nearest even, at most half a step (2^-4 of the value) off;
 *   magnitudes above 448 * 2^119 = 2.98e38 are held as that;
 *   infinities and NaN become the format's NaN and change no other value of the row.
 *   value = code * 2^(byte - 127)
 * A power of two costs a floating format no precision, the division by it is exact, and every value is exact in bf16
 * as well as fp32, so that the chip's conversions and matrix instructions add no error of their own.
 *
 * Conventions are those of emm.h.  dtype of the batch is that of q, k_new, v_new, out and of what is read back; the
 * pools' are fixed.  Slots that hold no token may hold any bits.  emm_kv_pages_pack / emm_kv_pages_unpack move pages
 * of the code pools (page_bytes = num_kv_heads * page_size * head_dim) and, in a call of their own, of the scale pools
 * (num_kv_heads * page_size) as they are.
 *
 * Limits of these calls and of emm_rope (beyond them EMM_ERR_UNSUPPORTED): 2^25 tokens and 2^30 (token, head) rows in
 * a batch, 4096 heads, 2^30 slots in a row of the page table; for the attention, 2^20 (request, KV head) pairs.
 */
#ifndef EMM_FP8_H
#define EMM_FP8_H

#include "emm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The pools, device memory, 16-byte aligned.  num_pages is the batch's. */
typedef struct {
    void *k, *v;                 /* [num_pages][num_kv_heads][page_size][head_dim] codes             */
    void *k_scale, *v_scale;     /* [num_pages][num_kv_heads][page_size] scale bytes                 */
} emm_fp8_cache;

/*
 * emm_kv_scatter into such a cache: the new tokens' K and V rows are quantised on the way.  token_stride as for
 * emm_rope (0: k_new and v_new are packed; else elements from a token's row to the next in both).  EMM_BF16 or
 * EMM_F32, head_dim 64 or 128.  No other byte of the pools is written.
 */
emm_status emm_kv_scatter_fp8(const emm_batch *batch, const void *k_new, const void *v_new, int64_t token_stride,
                              const emm_fp8_cache *cache, void *hip_stream);

/*
 * emm_rope and emm_kv_scatter_fp8 in one launch, with the bits of the two: q is rotated into q_out (packed; may be q
 * where that is packed), k_new is rotated, rounded to the batch's dtype and quantised, v_new is quantised.
 * token_stride holds for q, k_new and v_new.  As by emm_rope, q's rows of no request are turned where positions are
 * given, and else left as they were.
 */
emm_status emm_rope_kv_scatter_fp8(const emm_batch *batch, const emm_rope_params *rope, const void *q, const void *k_new,
                                   const void *v_new, int64_t token_stride, void *q_out, const emm_fp8_cache *cache,
                                   void *hip_stream);

/*
 * Reads slots back, the inverse of emm_kv_scatter_fp8: k_out[cu_new_lens[r] + j][h] (packed, the batch's dtype) is
 * the value of slot prefix_lens[r] + j of request r; so prefix_lens 0 and new_lens the contexts' lengths give whole
 * contexts.  Exact in both dtypes.  EMM_BF16 or EMM_F32, head_dim 64 or 128.  Rows of no request are left as they were.
 */
emm_status emm_kv_gather_fp8(const emm_batch *batch, const emm_fp8_cache *cache, void *k_out, void *v_out, void *hip_stream);

/*
 * emm_prefill_attn, emm_cross_attn and emm_decode_attn over such a cache: the attention of the values that it stands
 * for, for any number of new tokens per request (emm_decode_attn_fp8: at most one, else EMM_ERR_INVALID_ARG).
 * EMM_BF16 with head_dim 128.  Arguments and results as there.  Values are exact in bf16 and meet q as such; scores,
 * softmax statistics and sums are in 32 bits; softmax weights are rounded to bf16 for the value product.  A NaN in V
 * reaches only rows that see its slot.  Results are run-to-run bitwise deterministic.
 * The sums are divided by the sum of the weights at the end, and weights are at most 2^16 on average until then: results
 * are finite where 2^16 * (slots of the context) * (largest |v|) is at most 2^127, so in a context of 2^17 slots for |v|
 * up to 2^94.  Larger values, which the format holds, may come out as infinities or NaN.
 *   workspace  device scratch of at least emm_attn_fp8_workspace_size bytes, 16-byte aligned (may be NULL if that is
 *              0), the same size for all three calls; contents need no initialisation and mean nothing afterwards.
 *              Calls that may overlap must not share one.
 */
emm_status emm_attn_fp8_workspace_size(const emm_batch *batch, size_t *bytes);
emm_status emm_prefill_attn_fp8(const emm_batch *batch, const void *q, const emm_fp8_cache *cache, void *out, float *lse,
                                void *workspace, size_t workspace_bytes, void *hip_stream);
emm_status emm_cross_attn_fp8(const emm_batch *batch, const void *q, const emm_fp8_cache *cache, void *out, float *lse,
                              void *workspace, size_t workspace_bytes, void *hip_stream);
emm_status emm_decode_attn_fp8(const emm_batch *batch, const void *q, const emm_fp8_cache *cache, void *out, float *lse,
                               void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* EMM_FP8_H */
