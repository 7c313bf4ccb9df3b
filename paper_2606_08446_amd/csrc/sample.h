// Launcher of the token sampler (sample.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sparrow {

constexpr int kSampleMaxVocab = SPARROW_SAMPLE_MAX_VOCAB;

struct SampleArgs {
    const void *logits;
    int64_t row_stride;  // elements from row to row
    int64_t rows;
    int vocab;
    bool bf16;
    const float *temperature;  // null: 1
    const int32_t *top_k;      // null: off (as are the next two)
    const float *top_p, *min_p;
    const float *uniform;
    int32_t *tokens;
    float *logprobs;  // null: not wanted
};

size_t sample_workspace(int64_t rows, int vocab, bool bf16);
hipError_t launch_sample(const SampleArgs &a, void *workspace, hipStream_t stream);

}  // namespace sparrow
