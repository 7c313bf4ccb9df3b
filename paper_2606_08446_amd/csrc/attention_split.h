// Parts of the decode attention's work split that do not depend on what the cache holds: the
// kernels' arguments, the page offsets of the sequences and the merge of partials.  attention.hip
// streams bf16 caches, attention_e4m3.hip 8-bit ones.
#pragma once

#include "common.h"
#include "wave.h"

namespace sparrow {

constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = kAttnThreads / 64;
constexpr int kBatch = 64;        // pages per prefetched page-list batch
constexpr int kMaxWaves = 4096;   // upper bound of streaming waves (sizes the workspace)

struct AttnArgs {
    const uint16_t *q;
    const uint16_t *k_cache;
    const uint16_t *v_cache;
    const int32_t *block_table;
    const int32_t *seq_lens;
    const int32_t *ksel;
    const int32_t *idx;
    int32_t *plan_off;    // [batch + 1] page offsets of the sequences (written by workgroup 0)
    int32_t *unit_waves;  // [batch * num_kv_heads][2] first and last wave of each unit
    float *o_part;
    float *ml_part;
    void *out;
    int k_max, batch, num_q_heads, num_kv_heads, ps, max_pages, out_bf16;
    int max_waves, fine_waves;  // streaming waves at most; and with single chunks (see k_attn_stream)
    int64_t num_phys;  // physical pages in the caches
    float scale_log2;
};

// Joins the partials that streaming waves left in the workspace; one launch.
hipError_t launch_attn_merge(const AttnArgs &a, hipStream_t stream);

namespace {

// Element `c` (0..7) of two 8 x bf16 vectors, packed as (x[c], y[c]).
__device__ __forceinline__ uint32_t pair_of(u32x4_t x, u32x4_t y, int c)
{
    const uint32_t a = x[c >> 1], b = y[c >> 1];
    return (c & 1) ? __builtin_amdgcn_perm(b, a, 0x07060302u)
                   : __builtin_amdgcn_perm(b, a, 0x05040100u);
}

__device__ __forceinline__ void store_out(void *out, int out_bf16, int64_t i, float v)
{
    if (out_bf16)
        static_cast<uint16_t *>(out)[i] = (uint16_t)to_bf16_bits(v);
    else
        static_cast<float *>(out)[i] = v;
}

// Pages in the attention list of sequence b.
template <bool kSparse>
__device__ __forceinline__ int list_pages(const AttnArgs &a, int b)
{
    const int L = clamp_len(a.seq_lens[b], a.ps, a.max_pages);
    const int n = (L + a.ps - 1) / a.ps;
    if (!kSparse)
        return n;
    const int c = a.ksel[b];
    return c < 0 ? 0 : (c > a.k_max ? a.k_max : c);
}

// Block-wide exclusive prefix of list_pages over the batch into s_off[0 .. batch].
template <bool kSparse>
__device__ void seq_prefix(const AttnArgs &a, int32_t *s_off, int32_t *s_tmp)
{
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = tid >> 6;
    const int B = a.batch;
    const int per = (B + kAttnThreads - 1) / kAttnThreads;
    const int b0 = min(B, tid * per);
    const int b1 = min(B, b0 + per);
    int local = 0;
    for (int b = b0; b < b1; ++b)
        local += list_pages<kSparse>(a, b);
    const int incl = (int)wave_scan_add((uint32_t)local);  // totals < 2^31 (max batch x pages)
    if (lane == 63)
        s_tmp[wave] = incl;
    __syncthreads();
    int run = incl - local;
    for (int w = 0; w < wave; ++w)
        run += s_tmp[w];
    for (int b = b0; b < b1; ++b) {
        s_off[b] = run;
        run += list_pages<kSparse>(a, b);
    }
    if (tid == kAttnThreads - 1)
        s_off[B] = run;  // this thread's range ends at B (or is empty): run is the total
    __syncthreads();
}

}  // namespace
}  // namespace sparrow
