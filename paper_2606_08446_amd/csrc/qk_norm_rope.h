// Launchers of the per-head norm with rotation (qk_norm_rope.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sparrow {

struct RopeArgs {
    const uint16_t *q, *k;  // input rows, `*_stride` elements from token to token
    int64_t q_stride, k_stride;
    const uint16_t *q_weight, *k_weight;
    const double *inv_freq;
    const int32_t *positions;
    int64_t tokens;
    int num_q_heads, num_k_heads;
    float eps;
};

struct RopeGradArgs {
    const uint16_t *dq_out, *dk_out;
    uint16_t *dq, *dk;
    int64_t dq_stride, dk_stride;
    float *dq_weight, *dk_weight;
    float *partials;  // [kRopeGradBlocks][128]
};

// Workgroups of the gradient at most: two per CU, so that the weights' partial sums stay few (256 /
// 512 / 1024: 32K tokens of 32 + 8 heads 203 / 171 / 186 us, 1014 of 40 + 8 heads 16.2 / 12.7 / 13.2).
constexpr int kRopeGradBlocks = 512;

hipError_t launch_qk_norm_rope(const RopeArgs &a, uint16_t *q_out, uint16_t *k_out,
                               hipStream_t stream);
hipError_t launch_qk_norm_rope_bwd(const RopeArgs &a, const RopeGradArgs &g, hipStream_t stream);

}  // namespace sparrow
