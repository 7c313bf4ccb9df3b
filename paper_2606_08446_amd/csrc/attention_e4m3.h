// Launcher of the decode attention over an e4m3 cache (attention_e4m3.hip).
#pragma once

#include "cache_e4m3.h"
#include "common.h"

namespace sparrow {

// idx != nullptr: over the page lists (k, idx, k_max); else over every page.
hipError_t launch_attention_e4m3(const sparrow_shape_t &s, const AttnPlan &plan, const void *q,
                                 const CacheE4m3 &c, const int32_t *block_table,
                                 const int32_t *seq_lens, const int32_t *k, const int32_t *idx,
                                 int32_t k_max, float scale, void *out, int out_dtype,
                                 void *workspace, hipStream_t stream);

}  // namespace sparrow
