// Launcher of the decode attention of groups with a shared prefix (attention_shared.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "sparrow.h"

namespace sparrow {

constexpr int kMaxGroups = SPARROW_MAX_GROUPS;

struct Groups {
    const int32_t *cu;      // [n + 1] first sequence of every group
    const int32_t *prefix;  // [n] tokens that a group's sequences share
    int n;
};

size_t shared_attention_workspace(const sparrow_shape_t &s, int groups);
hipError_t launch_shared_attention(const sparrow_shape_t &s, const Groups &g, const void *q,
                                   const void *k_cache, const void *v_cache,
                                   const int32_t *block_table, const int32_t *seq_lens, float scale,
                                   void *out, int out_dtype, void *workspace, hipStream_t stream);

}  // namespace sparrow
