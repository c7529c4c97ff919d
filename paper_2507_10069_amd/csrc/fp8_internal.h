// What the entry points of rotary positions and of the 8-bit cache hand to the kernels.
#pragma once

#include "emm_internal.h"

namespace emm {

constexpr long long MOST_SLOTS = 1ll << 30;  // in a row of the page table, for the calls of emm_fp8.h and emm_rope

// Rotary positions (see emm_rope_params): arrays of the device, ends[a] = frequencies of the axes up to a
struct RopeView {
    const double* inv_freq;
    const int32_t* positions;        // [num_axes][T], or nullptr: a token's place in its request
    int32_t rotary_dim;              // 0: nothing is rotated
    int32_t interleaved;
    int32_t num_axes;
    int32_t ends[3];
    float factor;
    float sine_factor;               // factor, with the sign of the inverse
};
// The 8-bit cache's pools (see emm_fp8_cache)
struct Fp8Pools {
    unsigned char *k, *v, *k_scale, *v_scale;
};
// Rows of a batch on their way: q (nullptr: none), k and v (nullptr: none) with the strides of their tokens' rows in elements
struct NewRows {
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    void *q_out, *k_out;             // packed
};
// rotates q into q_out, and k into k_out (pools: nullptr) or, quantised together with v, into the pools; rope.rotary_dim 0: no rotation
hipError_t launch_rope_rows(const BatchView& b, bool bf16, const RopeView& rope, const NewRows& rows, const Fp8Pools* pools, hipStream_t stream);
hipError_t launch_kv_gather_fp8(const BatchView& b, bool bf16, const Fp8Pools& pools, void* k_out, void* v_out, hipStream_t stream);

struct AttnFp8Args {
    BatchView b;
    const void* q;
    Fp8Pools pools;
    void* out;
    float* lse;
    void* workspace;
};
size_t attn_fp8_workspace_bytes(const BatchView& b);
size_t attn_fp8_tiles_workspace_bytes(const BatchView& b);
hipError_t launch_attn_fp8_tiles(const AttnFp8Args& a, bool causal, hipStream_t stream);
hipError_t launch_attn_fp8(const AttnFp8Args& a, bool causal, hipStream_t stream);

}  // namespace emm
