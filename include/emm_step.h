/*
 * emm_step.h -- a decoder layer's step around and in place of full attention: page tables and slots made on the device,
 * norms of q and k with rotation and cache write in one pass, attention with a window.  Together they are the step of a
 * model whose layers look back a fixed distance, in a loop that the host does not have to look into:
 *
 *   emm_page_step                                the step's tables, offsets, positions and slots from lengths
 *   emm_norm_rope_kv_scatter (or _fp8)           q and k normed and rotated, k and v into their slots
 *   emm_prefill_attn_window / emm_decode_attn_window   attention over the last `window` tokens and the first `sinks`
 *
 * Conventions are those of emm.h, and the limits on sizes those of emm_fp8.h: 2^25 tokens and 2^30 (token, head) rows in
 * a batch, 4096 heads, 2^30 slots in a row of the page table (beyond them EMM_ERR_UNSUPPORTED).
 */
#ifndef EMM_STEP_H
#define EMM_STEP_H

#include "emm.h"
#include "emm_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * One step's page tables from the lengths that requests have and the tokens they bring.  In this order, as if the
 * requests took their turns one after the other:
 *   1. Pages that no token of this step or a later one sees are given back.  With window > 0 the tokens of request r, the
 *      first of which is at slot c = lens[r], see the slots from c - window + 1 on and the first `sinks`; entries
 *      e = held_from[r] (at least ceil(sinks / page_size)), ... of its table whose page lies wholly before are pushed onto
 *      the stack of free pages, in order of r, then e.  held_out[r] is the first entry that it keeps of these; what the
 *      table says of entries before that means nothing any more (it is left as it was).  So entries 0 .. held_from[r] - 1
 *      are never given back: start at the pages that are shared with others (a cached prefix), or 0.
 *      With window == 0 nothing is given back, and held_out is held_from (at least the sinks' pages).
 *   2. A request that brings m = add_lens[r] tokens gets ceil((c + m) / page_size) - ceil(c / page_size) pages, popped from
 *      the stack one by one into the next entries of its table.  A request whose tokens do not fit its row of the table, or
 *      that finds too few pages, or that needs pages after one that found too few, is refused: it takes none and brings
 *      none.  *refused counts those that have tokens.
 *   3. prefix_lens[r] = c, new_lens[r] = m or 0 (refused), cu_new_lens = the running sum, lens_out[r] = c + new_lens[r]: the
 *      arrays of an emm_batch and, for every token t of request r, positions[t] = its slot in the request and slots[t] = its
 *      slot in the pool, page_table[r][position / page_size] * page_size + position % page_size.  Behind the last token
 *      up to max_tokens: slots[t] = -1, positions[t] = 0.
 * Each output may be the input that it follows (lens_out = lens, held_out = held_from, free_count_out = free_count): so one
 * captured graph is a loop's every step.  Otherwise inputs and outputs do not overlap; page_table and free_pages are read
 * and written.  Where they are kept apart the step can be done again: no entry that it reads is written, whatever it takes
 * or gives back (so a refused step is repeated when pages have been pushed).
 * The caller sees to it that add_lens add up to at most max_tokens (what is beyond is left out of slots and positions), that lens
 * and tables are consistent and free_pages[0 .. *free_count - 1] are distinct and in no table; inconsistent arrays give
 * meaningless results but no access outside the buffers.  A negative add_lens is 0.  Whole numbers, the same on every run.
 */
typedef struct {
    int32_t num_reqs;            /* B, at most 4096                                                  */
    int32_t page_size;           /* 16, 32, 64, 128 or 256                                           */
    int32_t num_pages;           /* pages in each pool, at most 2^28                                 */
    int32_t max_pages_per_req;   /* row stride of page_table                                         */
    int32_t max_tokens;          /* T of the batch: entries of slots and positions                   */
    int32_t window;              /* 0: nothing is given back                                         */
    int32_t sinks;               /* >= 0                                                             */
    int32_t reserved;            /* must be 0                                                        */
    int32_t *page_table;         /* device [B][max_pages_per_req], read and written                  */
    int32_t *free_pages;         /* device [num_pages], a stack, read and written                    */
    const int32_t *lens;         /* device [B] tokens in the pages                                   */
    const int32_t *add_lens;     /* device [B] tokens that the step brings                           */
    const int32_t *held_from;    /* device [B]                                                       */
    const int32_t *free_count;   /* device [1] free pages                                            */
    int32_t *prefix_lens, *new_lens, *cu_new_lens;   /* device [B], [B], [B + 1]                     */
    int32_t *lens_out, *held_out, *free_count_out;   /* device [B], [B], [1]                         */
    int64_t *slots;              /* device [T], or NULL                                              */
    int32_t *positions;          /* device [T], or NULL                                              */
    int32_t *refused;            /* device [1], or NULL                                              */
} emm_page_step_params;
emm_status emm_page_step(const emm_page_step_params *step, void *hip_stream);

/*
 * Norms of q's and k's heads.  Each row x of a (token, head) becomes x / sqrt(mean(x^2) + eps) * weight, channel by channel,
 * with q's or k's weights (the same for all heads).  In 32 bits; rows whose squares pass their range (|x| from 1.8e19 on)
 * come out right all the same.
 */
typedef struct {
    float eps;                   /* 1.2e-38 (the least normal number) or more                        */
    int32_t reserved;            /* must be 0                                                        */
    const float *q_weight;       /* device [head_dim], 16-byte aligned                               */
    const float *k_weight;       /* device [head_dim], 16-byte aligned                               */
} emm_qk_norm;

/*
 * emm_rope with the norm before the rotation, in one pass: normed, rotated, rounded once to the batch's dtype.  Arguments as
 * for emm_rope; norm or rope may be NULL (not both) and is left out then.  Of the batch's arrays none are read unless the
 * positions come from them (rope with num_axes 0: rows of no request are left as they were); else all T rows are done.
 */
emm_status emm_norm_rope(const emm_batch *batch, const emm_qk_norm *norm, const emm_rope_params *rope, const void *q, const void *k,
                         int64_t token_stride, void *q_out, void *k_out, void *hip_stream);

/*
 * The same with the write of K and V into their slots: q becomes q_out (packed; may be q where that is packed), k_new is normed,
 * rotated and rounded on its way into k_cache, v_new is copied bit for bit into v_cache.  EMM_BF16 or EMM_F32, head_dim 64 or
 * 128.  token_stride holds for q, k_new and v_new.
 *   slots  device [T], 8-byte aligned: the slot in the pool of every token's K and V, distinct; none is written for a slot
 *          outside 0 .. num_pages * page_size - 1 (-1, say).  NULL: as emm_kv_scatter finds them, none for rows of no request.
 * q's rows of no request are done unless the positions come from the batch, as by emm_norm_rope.  No other byte of the
 * pools is written.
 * emm_norm_rope_kv_scatter_fp8 quantises the rows that emm_norm_rope would give as emm_kv_scatter_fp8 does, with the same bits.
 */
emm_status emm_norm_rope_kv_scatter(const emm_batch *batch, const emm_qk_norm *norm, const emm_rope_params *rope, const void *q,
                                    const void *k_new, const void *v_new, int64_t token_stride, const int64_t *slots, void *q_out,
                                    void *k_cache, void *v_cache, void *hip_stream);
emm_status emm_norm_rope_kv_scatter_fp8(const emm_batch *batch, const emm_qk_norm *norm, const emm_rope_params *rope, const void *q,
                                        const void *k_new, const void *v_new, int64_t token_stride, const int64_t *slots, void *q_out,
                                        const emm_fp8_cache *cache, void *hip_stream);

/*
 * emm_prefill_attn and emm_decode_attn with a window: new token j of request r, at slot p = prefix_lens[r] + j, sees the slots
 * k <= p with p - k < window (itself among them) or k < sinks.  window >= 1, sinks >= 0; a window of the context's length or
 * more is the full attention.
 * Entries of the page table whose page no new token sees are not looked at, so those pages may have been given back
 * (emm_page_step).  What a slot holds that a row does not see never reaches the row, infinities and NaN included.
 * One of them in V at a slot that the row sees makes that channel of the row infinite or NaN, whatever the slot's weight.
 * Arguments and results otherwise as for emm_prefill_attn (emm_decode_attn_window: at most one new token per request, else
 * EMM_ERR_INVALID_ARG); EMM_BF16 with head_dim 128 and EMM_F32 with head_dim 64 or 128; at most 2^20 (request, KV head) pairs.
 * bf16: scores, softmax statistics and sums in 32 bits; softmax weights are rounded to bf16 for the value product.  The sums are
 * divided by the sum of the weights at the end, and weights are at most 2^16 until then: results are finite where
 * 2^16 * (slots that the row sees) * (largest |v|) is at most 2^127.  Results are run-to-run bitwise deterministic.
 *   workspace  device scratch of at least emm_attn_window_workspace_size bytes, 16-byte aligned (may be NULL if that is 0), the
 *              same size for both calls; contents need no initialisation and mean nothing afterwards.  Calls that may overlap
 *              must not share one.
 */
emm_status emm_attn_window_workspace_size(const emm_batch *batch, int32_t window, int32_t sinks, size_t *bytes);
emm_status emm_prefill_attn_window(const emm_batch *batch, int32_t window, int32_t sinks, const void *q, const void *k_cache,
                                   const void *v_cache, void *out, float *lse, void *workspace, size_t workspace_bytes,
                                   void *hip_stream);
emm_status emm_decode_attn_window(const emm_batch *batch, int32_t window, int32_t sinks, const void *q, const void *k_cache,
                                  const void *v_cache, void *out, float *lse, void *workspace, size_t workspace_bytes,
                                  void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* EMM_STEP_H */
