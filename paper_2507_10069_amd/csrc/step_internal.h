// What the entry points of emm_step.h hand to the kernels.
#pragma once

#include "fp8_internal.h"

namespace emm {

constexpr int MOST_STEP_REQS = 4096;         // requests of a page step: what its workgroups hold of each fits LDS
constexpr int MOST_STEP_PAGES = 1 << 28;     // pages in a pool of a page step (2 KB each would fill 512 GB); its sums stop at this

struct PageStepArgs {
    int32_t num_reqs, page_shift /* page size 16 << page_shift */, num_pages, max_pages, max_tokens, window, sink_pages;
    int32_t* page_table;
    int32_t* free_pages;
    const int32_t *lens, *add_lens, *held_from, *free_count;
    int32_t *prefix_lens, *new_lens, *cu_new_lens, *lens_out, *held_out, *free_count_out;
    int64_t* slots;
    int32_t *positions, *refused;
};
// in_place: an output is the input that it follows
hipError_t launch_page_step(const PageStepArgs& a, bool in_place, hipStream_t stream);

// Norms of q's and k's rows (see emm_qk_norm) and given slots
struct NormView {
    const float *q_weight, *k_weight;        // nullptr: no norm
    float eps;
    const int64_t* slots;                    // [T], or nullptr: from the batch
};
// the pools of a cache in the batch's dtype
struct PlainPools {
    void *k, *v;
};
// As launch_rope_rows, with the norm before the rotation.  At most one of fp8 and plain.
hipError_t launch_norm_rope_rows(const BatchView& b, bool bf16, const NormView& norm, const RopeView& rope, const NewRows& rows, const Fp8Pools* fp8,
                                 const PlainPools* plain, hipStream_t stream);

// What a row sees besides keys up to its own place: those less than `window` before it, and the first `sinks`
struct WindowView {
    int32_t window, sinks;
};
// the slots behind the sinks that the token at slot p does not see any more: those before this one
__host__ __device__ inline int window_low(const WindowView& w, int p) { return p - w.window + 1 > 0 ? p - w.window + 1 : 0; }

hipError_t launch_attn_f32_window(const AttnArgs& a, const WindowView& w, hipStream_t stream);
size_t attn_window_workspace_bytes(const BatchView& b, const WindowView& w);
hipError_t launch_attn_window(const AttnArgs& a, const WindowView& w, hipStream_t stream);

}  // namespace emm
