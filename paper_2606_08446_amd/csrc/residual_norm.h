// Launchers of the norms around a block (residual_norm.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sparrow {

constexpr int kNormMaxChannels = 16384;

struct NormArgs {
    const void *h;              // the stream, bf16 or fp32 [tokens][channels]
    const uint16_t *x, *gate;   // the block's output and its gate's logits (null: none)
    int64_t x_stride, gate_stride;
    const uint16_t *weight, *post;
    int64_t tokens;
    int channels;
    bool f32;  // the stream's type
    float scale, eps;
};

struct NormGradArgs {
    const uint16_t *dy;
    const void *dh_out;  // null: zero
    void *dh;
    uint16_t *dx, *dgate;
    int64_t dx_stride, dgate_stride;
    float *dweight, *dpost;
    float *partials;  // [norm_grad_blocks][1 or 2][channels]
};

// Workgroups of the gradient: a function of the sizes alone, so that its sums are too.
int norm_grad_blocks(int64_t tokens, int channels);
size_t norm_grad_workspace(int64_t tokens, int channels);

hipError_t launch_residual_norm(const NormArgs &a, void *h_out, uint16_t *y, hipStream_t stream);
hipError_t launch_residual_norm_bwd(const NormArgs &a, const NormGradArgs &g, hipStream_t stream);

}  // namespace sparrow
