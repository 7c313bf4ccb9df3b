// C ABI of libsparrow: argument validation, workspace sizing and kernel launches.
// Declarations and the contract of every entry point are in include/sparrow.h.
#include <cmath>

#include "attention_e4m3.h"
#include "attention_shared.h"
#include "cache_e4m3.h"
#include "common.h"
#include "qk_norm_rope.h"
#include "residual_norm.h"
#include "sample.h"

using namespace sparrow;

namespace {

int check_shape(const sparrow_shape_t *s)
{
    if (!s)
        return SPARROW_EINVAL;
    if (s->batch < 0 || s->num_q_heads < 1 || s->num_kv_heads < 1 || s->max_pages_per_seq < 1 ||
        s->num_phys_pages < 1)
        return SPARROW_EINVAL;
    if (s->num_q_heads % s->num_kv_heads != 0)
        return SPARROW_EINVAL;
    if (s->num_q_heads / s->num_kv_heads > 16)
        return SPARROW_EUNSUPPORTED;
    if (s->head_dim != kHeadDim)
        return SPARROW_EUNSUPPORTED;
    if (s->page_size != 16 && s->page_size != 32 && s->page_size != 64 && s->page_size != 128)
        return SPARROW_EUNSUPPORTED;
    if (s->max_pages_per_seq > SPARROW_MAX_PAGES_PER_SEQ)
        return SPARROW_EUNSUPPORTED;
    if (s->landmark != SPARROW_LANDMARK_MINMAX && s->landmark != SPARROW_LANDMARK_MEAN)
        return SPARROW_EUNSUPPORTED;
    if ((int64_t)s->batch * s->num_q_heads > 0x7fffffff / kHeadDim)
        return SPARROW_EINVAL;
    return SPARROW_OK;
}

// The kernels move bf16/fp32 data in 16-byte vectors and indices as int32.
bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool al4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int status_of(hipError_t e) { return e == hipSuccess ? SPARROW_OK : SPARROW_EHIP; }

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// sparrow_decode_step's workspace: the scores, then the attention's workspace.
size_t decode_step_workspace(const sparrow_shape_t &s)
{
    return round256(score_topk_workspace(s)) + plan_attention(s).workspace_bytes;
}

bool al8(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

// Token strides of rows of `heads` heads: rows may not overlap and start on 16 bytes.
bool row_stride_ok(int64_t stride, int heads)
{
    return stride % 8 == 0 && stride >= (int64_t)heads * kHeadDim;
}

// Shared by sparrow_qk_norm_rope and its gradient; fills `a` where the arguments are fine.
int rope_args(int64_t num_tokens, int32_t num_q_heads, int32_t num_k_heads, int32_t head_dim,
              const void *q, int64_t q_stride, const void *k, int64_t k_stride,
              const void *q_weight, const void *k_weight, const double *inv_freq,
              const int32_t *positions, float eps, RopeArgs &a)
{
    if (num_tokens < 0 || num_tokens > 0x7fffffff || num_q_heads < 1 || num_k_heads < 1 ||
        num_q_heads > 1024 || num_k_heads > 1024)
        return SPARROW_EINVAL;
    if (head_dim != kHeadDim)
        return SPARROW_EUNSUPPORTED;
    if (!q || !k || !q_weight || !k_weight || !inv_freq || !positions)
        return SPARROW_EINVAL;
    if (!al16(q) || !al16(k) || !al16(q_weight) || !al16(k_weight) || !al8(inv_freq) ||
        !al4(positions))
        return SPARROW_EINVAL;
    if (!row_stride_ok(q_stride, num_q_heads) || !row_stride_ok(k_stride, num_k_heads) ||
        !(eps >= 0.f) || !std::isfinite(eps))
        return SPARROW_EINVAL;
    a = RopeArgs{static_cast<const uint16_t *>(q),        static_cast<const uint16_t *>(k),
                 q_stride,                                k_stride,
                 static_cast<const uint16_t *>(q_weight), static_cast<const uint16_t *>(k_weight),
                 inv_freq,                                positions,
                 num_tokens,                              num_q_heads,
                 num_k_heads,                             eps};
    return SPARROW_OK;
}

// Rows of `channels` bf16 values at any stride of whole 16-byte vectors.
bool rows_ok(const void *p, int64_t stride, int channels)
{
    return p && al16(p) && stride % 8 == 0 && stride >= channels;
}

// Shared by sparrow_residual_norm and its gradient (h: the stream that it reads); fills `a` where the
// arguments are fine.
int norm_args(int64_t num_tokens, int32_t channels, int32_t stream_dtype, const void *h,
              const void *x, int64_t x_stride, const void *gate, int64_t gate_stride,
              const void *weight, const void *post_weight, float scale, float eps, NormArgs &a)
{
    if (num_tokens < 0 || num_tokens > 0x7fffffff || channels < 8)
        return SPARROW_EINVAL;
    if (channels % 8 || channels > kNormMaxChannels ||
        (stream_dtype != SPARROW_STREAM_F32 && stream_dtype != SPARROW_STREAM_BF16))
        return SPARROW_EUNSUPPORTED;
    if (!h || !weight || !al16(h) || !al16(weight) || !al16(post_weight))
        return SPARROW_EINVAL;
    if ((x && !rows_ok(x, x_stride, channels)) || (gate && !rows_ok(gate, gate_stride, channels)))
        return SPARROW_EINVAL;
    if (!std::isfinite(scale) || !(eps >= 0.f) || !std::isfinite(eps))
        return SPARROW_EINVAL;
    a = NormArgs{h,
                 static_cast<const uint16_t *>(x),
                 static_cast<const uint16_t *>(gate),
                 x_stride,
                 gate_stride,
                 static_cast<const uint16_t *>(weight),
                 static_cast<const uint16_t *>(post_weight),
                 num_tokens,
                 channels,
                 stream_dtype == SPARROW_STREAM_F32,
                 scale,
                 eps};
    return SPARROW_OK;
}

// Rows of new (or read) tokens of an e4m3 cache.
int check_rows(const sparrow_shape_t &s, const int32_t *cu_tokens, int64_t num_tokens)
{
    if (num_tokens < 0 || num_tokens > (1 << 27) || !al4(cu_tokens))
        return SPARROW_EINVAL;
    if (cu_tokens == nullptr && num_tokens != s.batch)
        return SPARROW_EINVAL;
    if (s.num_kv_heads > 65535 || s.batch > (1 << 20))  // grid dimensions
        return SPARROW_EINVAL;
    return SPARROW_OK;
}

// Shared by the two attention calls over an e4m3 cache (dense: k and idx are null, k_max 0).
int attention_e4m3_call(bool sparse, const sparrow_shape_t *shape, const void *q,
                        const void *k_cache, const void *v_cache, const void *exps,
                        const int32_t *block_table, const int32_t *seq_lens, const int32_t *k,
                        const int32_t *idx, int32_t k_max, float scale, void *out,
                        int32_t out_dtype, void *workspace, size_t ws_bytes, void *stream)
{
    const int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    if (!q || !k_cache || !v_cache || !exps || !block_table || !seq_lens || !out ||
        (sparse && (!k || !idx)))
        return SPARROW_EINVAL;
    if (!al16(q) || !al16(k_cache) || !al16(v_cache) || !al8(exps) || !al4(block_table) ||
        !al4(seq_lens) || !al4(k) || !al4(idx) || !al16(out) || !al16(workspace))
        return SPARROW_EINVAL;
    if (sparse && (k_max < 1 || k_max > SPARROW_MAX_PAGES_PER_SEQ))
        return SPARROW_EINVAL;
    if (out_dtype != SPARROW_OUT_F32 && out_dtype != SPARROW_OUT_BF16)
        return SPARROW_EUNSUPPORTED;
    if (shape->batch == 0)
        return SPARROW_OK;
    // (the kernels number the cache's 16-token parts in 32 bits: 4 TiB of codes)
    if (shape->batch > kMaxBatch ||
        shape->num_phys_pages > 0x7fffffff / (shape->page_size / 16) / shape->num_kv_heads)
        return SPARROW_EUNSUPPORTED;
    const AttnPlan plan = plan_attention(*shape);
    if (!workspace || ws_bytes < plan.workspace_bytes)
        return SPARROW_EWORKSPACE;
    // (the kernels only read the cache)
    const CacheE4m3 cache{static_cast<uint8_t *>(const_cast<void *>(k_cache)),
                          static_cast<uint8_t *>(const_cast<void *>(v_cache)),
                          static_cast<uint8_t *>(const_cast<void *>(exps))};
    return status_of(launch_attention_e4m3(*shape, plan, q, cache, block_table, seq_lens, k, idx,
                                           k_max, scale, out, out_dtype, workspace,
                                           static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int sparrow_page_meta_update(const sparrow_shape_t *shape, const void *k_cache,
                             const int32_t *block_table, const int32_t *seq_lens,
                             const int32_t *first_pos, void *meta, void *stream)
{
    const int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    if (!k_cache || !block_table || !seq_lens || !meta)
        return SPARROW_EINVAL;
    if (!al16(k_cache) || !al16(meta) || !al4(block_table) || !al4(seq_lens) || !al4(first_pos))
        return SPARROW_EINVAL;
    if (shape->batch == 0)
        return SPARROW_OK;
    if (first_pos == nullptr && shape->batch > 65535)
        return SPARROW_EINVAL;
    return status_of(launch_meta_update(*shape, k_cache, block_table, seq_lens, first_pos, meta,
                                        static_cast<hipStream_t>(stream)));
}

int sparrow_append_kv(const sparrow_shape_t *shape, const void *k_new, const void *v_new,
                      void *k_cache, void *v_cache, const int32_t *block_table,
                      const int32_t *seq_lens, void *meta, void *stream)
{
    const int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    if (!k_new || !v_new || !k_cache || !v_cache || !block_table || !seq_lens || !meta)
        return SPARROW_EINVAL;
    if (!al16(k_new) || !al16(v_new) || !al16(k_cache) || !al16(v_cache) || !al16(meta) ||
        !al4(block_table) || !al4(seq_lens))
        return SPARROW_EINVAL;
    if (shape->batch == 0)
        return SPARROW_OK;
    return status_of(launch_append_kv(*shape, k_new, v_new, k_cache, v_cache, block_table,
                                      seq_lens, meta, static_cast<hipStream_t>(stream)));
}

// Shared by sparrow_page_score_topk and sparrow_append_score_topk.
static int score_topk_call(const sparrow_shape_t *shape, const void *q, void *meta,
                           const int32_t *block_table, const int32_t *seq_lens,
                           const sparrow_schedule_t *schedule, int32_t k_max, int32_t *out_k,
                           int32_t *out_idx, void *workspace, size_t ws_bytes,
                           const AppendArgs &app, void *stream)
{
    const int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    if (!q || !meta || !block_table || !seq_lens || !schedule || !out_k || !out_idx)
        return SPARROW_EINVAL;
    if (!al16(q) || !al16(meta) || !al4(block_table) || !al4(seq_lens) || !al4(out_k) ||
        !al4(out_idx) || !al16(workspace))
        return SPARROW_EINVAL;
    if (k_max < 1 || k_max > SPARROW_MAX_PAGES_PER_SEQ || schedule->bin_tokens < 1 || schedule->n_bins < 1 || schedule->frac_den < 1 ||
        !schedule->min_pages || !schedule->frac_num || schedule->sink_pages < 0 ||
        schedule->local_pages < 0)
        return SPARROW_EINVAL;
    if (shape->batch == 0)
        return SPARROW_OK;
    if ((int64_t)shape->batch * shape->num_kv_heads > 65535)
        return SPARROW_EINVAL;
    if (shape->batch > kMaxBatch)
        return SPARROW_EUNSUPPORTED;
    if (!workspace || ws_bytes < score_topk_workspace(*shape))
        return SPARROW_EWORKSPACE;
    Sched sched{schedule->bin_tokens, schedule->n_bins,     schedule->frac_den,
                schedule->min_pages,  schedule->frac_num, schedule->sink_pages,
                schedule->local_pages};
    return status_of(launch_score_topk(*shape, q, meta, block_table, seq_lens, sched, k_max,
                                       out_k, out_idx, workspace, app,
                                       static_cast<hipStream_t>(stream)));
}

int sparrow_page_score_topk(const sparrow_shape_t *shape, const void *q, const void *meta,
                            const int32_t *block_table, const int32_t *seq_lens,
                            const sparrow_schedule_t *schedule, int32_t k_max, int32_t *out_k,
                            int32_t *out_idx, void *workspace, size_t ws_bytes, void *stream)
{
    const AppendArgs none{nullptr, nullptr, nullptr, nullptr};
    // Without an append the kernel only reads the metadata.
    return score_topk_call(shape, q, const_cast<void *>(meta), block_table, seq_lens, schedule,
                           k_max, out_k, out_idx, workspace, ws_bytes, none, stream);
}

int sparrow_append_score_topk(const sparrow_shape_t *shape, const void *q, const void *k_new,
                              const void *v_new, void *k_cache, void *v_cache, void *meta,
                              const int32_t *block_table, const int32_t *seq_lens,
                              const sparrow_schedule_t *schedule, int32_t k_max, int32_t *out_k,
                              int32_t *out_idx, void *workspace, size_t ws_bytes, void *stream)
{
    const int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    if (!k_new || !v_new || !k_cache || !v_cache)
        return SPARROW_EINVAL;
    if (!al16(k_new) || !al16(v_new) || !al16(k_cache) || !al16(v_cache))
        return SPARROW_EINVAL;
    const AppendArgs app{k_new, v_new, k_cache, v_cache};
    return score_topk_call(shape, q, meta, block_table, seq_lens, schedule, k_max, out_k, out_idx,
                           workspace, ws_bytes, app, stream);
}

int sparrow_sparse_decode_attn(const sparrow_shape_t *shape, const void *q, const void *k_cache,
                               const void *v_cache, const int32_t *block_table,
                               const int32_t *seq_lens, const int32_t *k, const int32_t *idx,
                               int32_t k_max, float scale, void *out, int32_t out_dtype,
                               void *workspace, size_t ws_bytes, void *stream)
{
    const int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    if (!q || !k_cache || !v_cache || !block_table || !seq_lens || !k || !idx || !out)
        return SPARROW_EINVAL;
    if (!al16(q) || !al16(k_cache) || !al16(v_cache) || !al4(block_table) || !al4(seq_lens) ||
        !al4(k) || !al4(idx) || !al16(out) || !al16(workspace))
        return SPARROW_EINVAL;
    if (k_max < 1 || k_max > SPARROW_MAX_PAGES_PER_SEQ)
        return SPARROW_EINVAL;
    if (out_dtype != SPARROW_OUT_F32 && out_dtype != SPARROW_OUT_BF16)
        return SPARROW_EUNSUPPORTED;
    if (shape->batch == 0)
        return SPARROW_OK;
    if (shape->batch > kMaxBatch)
        return SPARROW_EUNSUPPORTED;
    const AttnPlan plan = plan_attention(*shape);
    if (!workspace || ws_bytes < plan.workspace_bytes)
        return SPARROW_EWORKSPACE;
    return status_of(launch_attention(*shape, plan, q, k_cache, v_cache, block_table, seq_lens, k,
                                      idx, k_max, scale, out, out_dtype, workspace,
                                      static_cast<hipStream_t>(stream)));
}

int sparrow_sparse_decode_attn_noalloc(const sparrow_shape_t *shape, const void *q,
                                       const void *k_cache, const void *v_cache,
                                       const int32_t *block_table, const int32_t *seq_lens,
                                       const int32_t *k, const int32_t *idx, int32_t k_max,
                                       float scale, void *out, int32_t out_dtype, void *stream)
{
    const int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    if (!q || !k_cache || !v_cache || !block_table || !seq_lens || !k || !idx || !out)
        return SPARROW_EINVAL;
    if (!al16(q) || !al16(k_cache) || !al16(v_cache) || !al4(block_table) || !al4(seq_lens) ||
        !al4(k) || !al4(idx) || !al16(out))
        return SPARROW_EINVAL;
    if (k_max < 1 || k_max > SPARROW_MAX_PAGES_PER_SEQ)
        return SPARROW_EINVAL;
    if (out_dtype != SPARROW_OUT_F32 && out_dtype != SPARROW_OUT_BF16)
        return SPARROW_EUNSUPPORTED;
    if (shape->batch == 0)
        return SPARROW_OK;
    if (shape->batch > kMaxBatch)
        return SPARROW_EUNSUPPORTED;
    const AttnPlan plan = plan_attention(*shape);
    if (plan.workspace_bytes > kScratchBytes)
        return SPARROW_EWORKSPACE;
    void *ws = attention_scratch();
    if (ws == nullptr)
        return SPARROW_EHIP;
    return status_of(launch_attention(*shape, plan, q, k_cache, v_cache, block_table, seq_lens, k,
                                      idx, k_max, scale, out, out_dtype, ws,
                                      static_cast<hipStream_t>(stream)));
}

int sparrow_dense_decode_attn(const sparrow_shape_t *shape, const void *q, const void *k_cache,
                              const void *v_cache, const int32_t *block_table,
                              const int32_t *seq_lens, float scale, void *out, int32_t out_dtype,
                              void *workspace, size_t ws_bytes, void *stream)
{
    const int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    if (!q || !k_cache || !v_cache || !block_table || !seq_lens || !out)
        return SPARROW_EINVAL;
    if (!al16(q) || !al16(k_cache) || !al16(v_cache) || !al4(block_table) || !al4(seq_lens) ||
        !al16(out) || !al16(workspace))
        return SPARROW_EINVAL;
    if (out_dtype != SPARROW_OUT_F32 && out_dtype != SPARROW_OUT_BF16)
        return SPARROW_EUNSUPPORTED;
    if (shape->batch == 0)
        return SPARROW_OK;
    if (shape->batch > kMaxBatch)
        return SPARROW_EUNSUPPORTED;
    const AttnPlan plan = plan_attention(*shape);
    if (!workspace || ws_bytes < plan.workspace_bytes)
        return SPARROW_EWORKSPACE;
    return status_of(launch_attention(*shape, plan, q, k_cache, v_cache, block_table, seq_lens,
                                      nullptr, nullptr, 0, scale, out, out_dtype, workspace,
                                      static_cast<hipStream_t>(stream)));
}

int sparrow_decode_step(const sparrow_shape_t *shape, const void *q, const void *k_new,
                        const void *v_new, void *k_cache, void *v_cache, void *meta,
                        const int32_t *block_table, const int32_t *seq_lens,
                        const sparrow_schedule_t *schedule, int32_t k_max, float scale,
                        int32_t *out_k, int32_t *out_idx, void *out, int32_t out_dtype,
                        void *workspace, size_t ws_bytes, void *stream)
{
    const int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    if (!q || !k_cache || !v_cache || !meta || !block_table || !seq_lens || !schedule || !out_k ||
        !out_idx || !out || (k_new == nullptr) != (v_new == nullptr))
        return SPARROW_EINVAL;
    if (!al16(q) || !al16(k_new) || !al16(v_new) || !al16(k_cache) || !al16(v_cache) ||
        !al16(meta) || !al4(block_table) || !al4(seq_lens) || !al4(out_k) || !al4(out_idx) ||
        !al16(out) || !al16(workspace))
        return SPARROW_EINVAL;
    if (k_max < 1 || k_max > SPARROW_MAX_PAGES_PER_SEQ || schedule->bin_tokens < 1 ||
        schedule->n_bins < 1 || schedule->frac_den < 1 || !schedule->min_pages ||
        !schedule->frac_num || schedule->sink_pages < 0 || schedule->local_pages < 0)
        return SPARROW_EINVAL;
    if (out_dtype != SPARROW_OUT_F32 && out_dtype != SPARROW_OUT_BF16)
        return SPARROW_EUNSUPPORTED;
    if (shape->batch == 0)
        return SPARROW_OK;
    if ((int64_t)shape->batch * shape->num_kv_heads > 65535)
        return SPARROW_EINVAL;
    if (shape->batch > kMaxBatch)
        return SPARROW_EUNSUPPORTED;
    if (!workspace || ws_bytes < decode_step_workspace(*shape))
        return SPARROW_EWORKSPACE;
    const Sched sched{schedule->bin_tokens, schedule->n_bins,     schedule->frac_den,
                      schedule->min_pages,  schedule->frac_num, schedule->sink_pages,
                      schedule->local_pages};
    const AppendArgs app{k_new, v_new, k_new ? k_cache : nullptr, k_new ? v_cache : nullptr};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    float *scores = static_cast<float *>(workspace);
    void *attn_ws = static_cast<char *>(workspace) + round256(score_topk_workspace(*shape));
    hipError_t e;
    if (attention_unit_path(*shape, k_max)) {
        if (score_select_path(*shape))
            return status_of(launch_decode_unit(*shape, q, k_cache, v_cache, meta, block_table,
                                                seq_lens, sched, k_max, out_k, out_idx, scale,
                                                out, out_dtype, app, st));
        e = launch_page_score(*shape, q, meta, block_table, seq_lens, sched, k_max, scores, app,
                              st);
        if (e != hipSuccess)
            return SPARROW_EHIP;
        return status_of(launch_select_attention(*shape, q, k_cache, v_cache, block_table,
                                                 seq_lens, sched, k_max, scores, out_k, out_idx,
                                                 scale, out, out_dtype, st));
    }
    e = launch_score_topk(*shape, q, meta, block_table, seq_lens, sched, k_max, out_k, out_idx,
                          scores, app, st);
    if (e != hipSuccess)
        return SPARROW_EHIP;
    return status_of(launch_attention(*shape, plan_attention(*shape), q, k_cache, v_cache,
                                      block_table, seq_lens, out_k, out_idx, k_max, scale, out,
                                      out_dtype, attn_ws, st));
}

int sparrow_shared_prefix_decode_attn(const sparrow_shape_t *shape, const void *q,
                                      const void *k_cache, const void *v_cache,
                                      const int32_t *block_table, const int32_t *seq_lens,
                                      int32_t num_groups, const int32_t *cu_groups,
                                      const int32_t *prefix_lens, float scale, void *out,
                                      int32_t out_dtype, void *workspace, size_t ws_bytes,
                                      void *stream)
{
    const int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    if (!q || !k_cache || !v_cache || !block_table || !seq_lens || !out || num_groups < 0 ||
        (num_groups > 0 && (!cu_groups || !prefix_lens)) || !std::isfinite(scale))
        return SPARROW_EINVAL;
    if (!al16(q) || !al16(k_cache) || !al16(v_cache) || !al4(block_table) || !al4(seq_lens) ||
        !al4(cu_groups) || !al4(prefix_lens) || !al16(out) || !al16(workspace))
        return SPARROW_EINVAL;
    if (out_dtype != SPARROW_OUT_F32 && out_dtype != SPARROW_OUT_BF16)
        return SPARROW_EUNSUPPORTED;
    if (shape->batch == 0)
        return SPARROW_OK;
    if ((int64_t)shape->batch * shape->num_kv_heads > 65535)
        return SPARROW_EINVAL;
    if (shape->batch > kMaxBatch || num_groups > kMaxGroups)
        return SPARROW_EUNSUPPORTED;
    if (!workspace || ws_bytes < shared_attention_workspace(*shape, num_groups))
        return SPARROW_EWORKSPACE;
    const Groups g{cu_groups, prefix_lens, num_groups};
    return status_of(launch_shared_attention(*shape, g, q, k_cache, v_cache, block_table, seq_lens,
                                             scale, out, out_dtype, workspace,
                                             static_cast<hipStream_t>(stream)));
}

size_t sparrow_shared_prefix_workspace_size(const sparrow_shape_t *shape, int32_t num_groups)
{
    if (check_shape(shape) != SPARROW_OK || shape->batch > kMaxBatch || num_groups < 0 ||
        num_groups > kMaxGroups || (int64_t)shape->batch * shape->num_kv_heads > 65535)
        return 0;
    return shared_attention_workspace(*shape, num_groups);
}

int sparrow_acceptance_rate(int64_t num_tokens, int32_t vocab, int32_t logits_dtype,
                            const void *target_logits, const void *draft_logits,
                            float inv_temperature, float *alpha, void *stream)
{
    if (num_tokens < 0 || vocab < 1 || !target_logits || !draft_logits || !alpha)
        return SPARROW_EINVAL;
    if (logits_dtype != SPARROW_LOGITS_F32 && logits_dtype != SPARROW_LOGITS_BF16)
        return SPARROW_EUNSUPPORTED;
    const uintptr_t esz = logits_dtype == SPARROW_LOGITS_BF16 ? 2 : 4;
    if ((reinterpret_cast<uintptr_t>(target_logits) % esz) != 0 ||
        (reinterpret_cast<uintptr_t>(draft_logits) % esz) != 0 || !al4(alpha))
        return SPARROW_EINVAL;
    // both rows of a token must share their alignment for the vector loads
    if ((reinterpret_cast<uintptr_t>(target_logits) & 15u) !=
        (reinterpret_cast<uintptr_t>(draft_logits) & 15u))
        return SPARROW_EINVAL;
    if (!std::isfinite(inv_temperature) || num_tokens > 0x7fffffff)
        return SPARROW_EINVAL;
    if (num_tokens == 0)
        return SPARROW_OK;
    return status_of(launch_acceptance(num_tokens, vocab, logits_dtype, target_logits,
                                       draft_logits, inv_temperature, alpha,
                                       static_cast<hipStream_t>(stream)));
}

int sparrow_acceptance_rate_topk(int64_t num_tokens, int32_t k, const float *lp_target,
                                 const float *lp_draft, float *alpha, void *stream)
{
    if (num_tokens < 0 || k < 1 || !lp_target || !lp_draft || !alpha)
        return SPARROW_EINVAL;
    if (!al4(lp_target) || !al4(lp_draft) || !al4(alpha))
        return SPARROW_EINVAL;
    if (num_tokens == 0)
        return SPARROW_OK;
    return status_of(launch_acceptance_topk(num_tokens, k, lp_target, lp_draft, alpha,
                                            static_cast<hipStream_t>(stream)));
}

int sparrow_sample(int64_t num_rows, int32_t vocab, int32_t logits_dtype, const void *logits,
                   int64_t row_stride, const float *temperature, const int32_t *top_k,
                   const float *top_p, const float *min_p, const float *uniform, int32_t *tokens,
                   float *logprobs, void *workspace, size_t ws_bytes, void *stream)
{
    if (num_rows < 0 || num_rows > 0x7fffffff || vocab < 1 || row_stride < vocab)
        return SPARROW_EINVAL;
    if (vocab > kSampleMaxVocab ||
        (logits_dtype != SPARROW_LOGITS_F32 && logits_dtype != SPARROW_LOGITS_BF16))
        return SPARROW_EUNSUPPORTED;
    const bool bf16 = logits_dtype == SPARROW_LOGITS_BF16;
    if (!logits || !uniform || !tokens ||
        (reinterpret_cast<uintptr_t>(logits) % (bf16 ? 2 : 4)) != 0 || !al4(temperature) ||
        !al4(top_k) || !al4(top_p) || !al4(min_p) || !al4(uniform) || !al4(tokens) ||
        !al4(logprobs) || !al16(workspace))
        return SPARROW_EINVAL;
    if (num_rows == 0)
        return SPARROW_OK;
    if (!workspace || ws_bytes < sample_workspace(num_rows, vocab, bf16))
        return SPARROW_EWORKSPACE;
    const SampleArgs a{logits, row_stride, num_rows, vocab,   bf16,   temperature,
                       top_k,  top_p,      min_p,    uniform, tokens, logprobs};
    return status_of(launch_sample(a, workspace, static_cast<hipStream_t>(stream)));
}

size_t sparrow_sample_workspace_size(int64_t num_rows, int32_t vocab, int32_t logits_dtype)
{
    if (num_rows < 0 || num_rows > 0x7fffffff || vocab < 1 || vocab > kSampleMaxVocab ||
        (logits_dtype != SPARROW_LOGITS_F32 && logits_dtype != SPARROW_LOGITS_BF16))
        return 0;
    return sample_workspace(num_rows, vocab, logits_dtype == SPARROW_LOGITS_BF16);
}

int sparrow_tail_stats(int64_t num_tokens, const float *alpha, const int32_t *positions,
                       int32_t bin_tokens, int32_t n_bins, double percentile, double *quantile,
                       double *mean, int64_t *count, void *stream)
{
    if (num_tokens < 0 || bin_tokens < 1 || n_bins < 1 || n_bins > 65535)
        return SPARROW_EINVAL;
    if (!(percentile >= 0.0 && percentile <= 100.0))
        return SPARROW_EINVAL;
    if (!quantile || !mean || !count || (num_tokens > 0 && (!alpha || !positions)))
        return SPARROW_EINVAL;
    if (!al4(alpha) || !al4(positions) || (reinterpret_cast<uintptr_t>(quantile) & 7u) ||
        (reinterpret_cast<uintptr_t>(mean) & 7u) || (reinterpret_cast<uintptr_t>(count) & 7u))
        return SPARROW_EINVAL;
    return status_of(launch_tail_stats(num_tokens, alpha, positions, bin_tokens, n_bins,
                                       percentile, quantile, mean, count,
                                       static_cast<hipStream_t>(stream)));
}

int sparrow_qk_norm_rope(int64_t num_tokens, int32_t num_q_heads, int32_t num_k_heads,
                         int32_t head_dim, const void *q, int64_t q_stride, const void *k,
                         int64_t k_stride, const void *q_weight, const void *k_weight,
                         const double *inv_freq, const int32_t *positions, float eps,
                         void *q_out, void *k_out, void *stream)
{
    RopeArgs a;
    const int rc = rope_args(num_tokens, num_q_heads, num_k_heads, head_dim, q, q_stride, k,
                             k_stride, q_weight, k_weight, inv_freq, positions, eps, a);
    if (rc != SPARROW_OK)
        return rc;
    if (!q_out || !k_out || !al16(q_out) || !al16(k_out))
        return SPARROW_EINVAL;
    if (num_tokens == 0)
        return SPARROW_OK;
    return status_of(launch_qk_norm_rope(a, static_cast<uint16_t *>(q_out),
                                         static_cast<uint16_t *>(k_out),
                                         static_cast<hipStream_t>(stream)));
}

int sparrow_qk_norm_rope_bwd(int64_t num_tokens, int32_t num_q_heads, int32_t num_k_heads,
                             int32_t head_dim, const void *dq_out, const void *dk_out,
                             const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                             const void *q_weight, const void *k_weight, const double *inv_freq,
                             const int32_t *positions, float eps, void *dq, int64_t dq_stride,
                             void *dk, int64_t dk_stride, float *dq_weight, float *dk_weight,
                             void *workspace, size_t ws_bytes, void *stream)
{
    RopeArgs a;
    const int rc = rope_args(num_tokens, num_q_heads, num_k_heads, head_dim, q, q_stride, k,
                             k_stride, q_weight, k_weight, inv_freq, positions, eps, a);
    if (rc != SPARROW_OK)
        return rc;
    if (!dq_out || !dk_out || !dq || !dk || !dq_weight || !dk_weight)
        return SPARROW_EINVAL;
    if (!al16(dq_out) || !al16(dk_out) || !al16(dq) || !al16(dk) || !al4(dq_weight) ||
        !al4(dk_weight) || !al16(workspace))
        return SPARROW_EINVAL;
    if (!row_stride_ok(dq_stride, num_q_heads) || !row_stride_ok(dk_stride, num_k_heads))
        return SPARROW_EINVAL;
    static_assert(sizeof(float) * kRopeGradBlocks * kHeadDim <= SPARROW_ROPE_WORKSPACE_BYTES,
                  "a row per workgroup");
    if (!workspace || ws_bytes < SPARROW_ROPE_WORKSPACE_BYTES)
        return SPARROW_EWORKSPACE;
    const RopeGradArgs g{static_cast<const uint16_t *>(dq_out),
                         static_cast<const uint16_t *>(dk_out),
                         static_cast<uint16_t *>(dq),
                         static_cast<uint16_t *>(dk),
                         dq_stride,
                         dk_stride,
                         dq_weight,
                         dk_weight,
                         static_cast<float *>(workspace)};
    return status_of(launch_qk_norm_rope_bwd(a, g, static_cast<hipStream_t>(stream)));
}

int sparrow_residual_norm(int64_t num_tokens, int32_t channels, int32_t stream_dtype, const void *h,
                          const void *x, int64_t x_stride, const void *gate, int64_t gate_stride,
                          const void *weight, const void *post_weight, float scale, float eps,
                          void *h_out, void *y, void *stream)
{
    NormArgs a;
    const int rc = norm_args(num_tokens, channels, stream_dtype, h, x, x_stride, gate, gate_stride,
                             weight, post_weight, scale, eps, a);
    if (rc != SPARROW_OK)
        return rc;
    if (!y || !al16(y) || !al16(h_out) || (x != nullptr) != (h_out != nullptr) ||
        (!x && (gate || post_weight)))
        return SPARROW_EINVAL;
    if (num_tokens == 0)
        return SPARROW_OK;
    return status_of(launch_residual_norm(a, h_out, static_cast<uint16_t *>(y),
                                          static_cast<hipStream_t>(stream)));
}

size_t sparrow_residual_norm_workspace_size(int64_t num_tokens, int32_t channels)
{
    if (num_tokens < 0 || num_tokens > 0x7fffffff || channels < 8 || channels % 8 ||
        channels > kNormMaxChannels)
        return 0;
    return norm_grad_workspace(num_tokens, channels);
}

int sparrow_residual_norm_bwd(int64_t num_tokens, int32_t channels, int32_t stream_dtype,
                              const void *dy, const void *dh_out, const void *h_out, const void *x,
                              int64_t x_stride, const void *gate, int64_t gate_stride,
                              const void *weight, const void *post_weight, float scale, float eps,
                              void *dh, void *dx, int64_t dx_stride, void *dgate,
                              int64_t dgate_stride, float *dweight, float *dpost_weight,
                              void *workspace, size_t ws_bytes, void *stream)
{
    NormArgs a;
    const int rc = norm_args(num_tokens, channels, stream_dtype, h_out, x, x_stride, gate,
                             gate_stride, weight, post_weight, scale, eps, a);
    if (rc != SPARROW_OK)
        return rc;
    if (!dy || !dh || !dweight || !al16(dy) || !al16(dh_out) || !al16(dh) || !al4(dweight) ||
        !al4(dpost_weight) || !al16(workspace))
        return SPARROW_EINVAL;
    if ((dx && !rows_ok(dx, dx_stride, channels)) ||
        (dgate && !rows_ok(dgate, dgate_stride, channels)))
        return SPARROW_EINVAL;
    if ((gate != nullptr) != (dgate != nullptr) ||
        (post_weight != nullptr) != (dpost_weight != nullptr) ||
        ((gate || post_weight) && (!x || !dx)))
        return SPARROW_EINVAL;
    if (num_tokens == 0)
        return SPARROW_OK;
    if (!workspace || ws_bytes < norm_grad_workspace(num_tokens, channels))
        return SPARROW_EWORKSPACE;
    if (!gate && !post_weight)
        a.x = nullptr;  // dx is then a multiple of dh
    const NormGradArgs g{static_cast<const uint16_t *>(dy),
                         dh_out,
                         dh,
                         static_cast<uint16_t *>(dx),
                         static_cast<uint16_t *>(dgate),
                         dx_stride,
                         dgate_stride,
                         dweight,
                         dpost_weight,
                         static_cast<float *>(workspace)};
    return status_of(launch_residual_norm_bwd(a, g, static_cast<hipStream_t>(stream)));
}

int sparrow_append_kv_e4m3(const sparrow_shape_t *shape, const void *k_new, int64_t k_stride,
                           const void *v_new, int64_t v_stride, const int32_t *cu_tokens,
                           int64_t num_tokens, void *k_cache, void *v_cache, void *exps,
                           const int32_t *block_table, const int32_t *seq_lens, void *meta,
                           void *stream)
{
    int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    rc = check_rows(*shape, cu_tokens, num_tokens);
    if (rc != SPARROW_OK)
        return rc;
    if (!k_new || !v_new || !k_cache || !v_cache || !exps || !block_table || !seq_lens || !meta)
        return SPARROW_EINVAL;
    if (!al16(k_new) || !al16(v_new) || !al16(k_cache) || !al16(v_cache) || !al8(exps) ||
        !al4(block_table) || !al4(seq_lens) || !al16(meta))
        return SPARROW_EINVAL;
    if (!row_stride_ok(k_stride, shape->num_kv_heads) ||
        !row_stride_ok(v_stride, shape->num_kv_heads))
        return SPARROW_EINVAL;
    if (shape->batch == 0 || num_tokens == 0)
        return SPARROW_OK;
    const NewRows rows{static_cast<const uint16_t *>(k_new), static_cast<const uint16_t *>(v_new),
                       k_stride, v_stride, cu_tokens, num_tokens};
    const CacheE4m3 cache{static_cast<uint8_t *>(k_cache), static_cast<uint8_t *>(v_cache),
                          static_cast<uint8_t *>(exps)};
    return status_of(launch_append_e4m3(*shape, rows, cache, block_table, seq_lens, meta,
                                        static_cast<hipStream_t>(stream)));
}

int sparrow_read_kv_e4m3(const sparrow_shape_t *shape, const void *k_cache, const void *v_cache,
                         const void *exps, const int32_t *block_table, const int32_t *seq_lens,
                         const int32_t *cu_tokens, int64_t num_tokens, void *k_out, void *v_out,
                         void *stream)
{
    int rc = check_shape(shape);
    if (rc != SPARROW_OK)
        return rc;
    rc = check_rows(*shape, cu_tokens, num_tokens);
    if (rc != SPARROW_OK)
        return rc;
    if (!k_cache || !v_cache || !exps || !block_table || !seq_lens || !k_out || !v_out)
        return SPARROW_EINVAL;
    if (!al16(k_cache) || !al16(v_cache) || !al8(exps) || !al4(block_table) || !al4(seq_lens) ||
        !al16(k_out) || !al16(v_out))
        return SPARROW_EINVAL;
    if (shape->batch == 0 || num_tokens == 0)
        return SPARROW_OK;
    // (the kernel only reads the cache)
    const CacheE4m3 cache{static_cast<uint8_t *>(const_cast<void *>(k_cache)),
                          static_cast<uint8_t *>(const_cast<void *>(v_cache)),
                          static_cast<uint8_t *>(const_cast<void *>(exps))};
    return status_of(launch_read_e4m3(*shape, cache, block_table, seq_lens, cu_tokens, num_tokens,
                                      k_out, v_out, static_cast<hipStream_t>(stream)));
}

int sparrow_sparse_decode_attn_e4m3(const sparrow_shape_t *shape, const void *q,
                                    const void *k_cache, const void *v_cache, const void *exps,
                                    const int32_t *block_table, const int32_t *seq_lens,
                                    const int32_t *k, const int32_t *idx, int32_t k_max,
                                    float scale, void *out, int32_t out_dtype, void *workspace,
                                    size_t ws_bytes, void *stream)
{
    return attention_e4m3_call(true, shape, q, k_cache, v_cache, exps, block_table, seq_lens, k,
                               idx, k_max, scale, out, out_dtype, workspace, ws_bytes, stream);
}

int sparrow_dense_decode_attn_e4m3(const sparrow_shape_t *shape, const void *q,
                                   const void *k_cache, const void *v_cache, const void *exps,
                                   const int32_t *block_table, const int32_t *seq_lens,
                                   float scale, void *out, int32_t out_dtype, void *workspace,
                                   size_t ws_bytes, void *stream)
{
    return attention_e4m3_call(false, shape, q, k_cache, v_cache, exps, block_table, seq_lens,
                               nullptr, nullptr, 0, scale, out, out_dtype, workspace, ws_bytes,
                               stream);
}

int sparrow_stream_read(const void *src, int64_t bytes, uint32_t *checksum, void *stream)
{
    if (bytes < 0 || (bytes & 15) != 0 || !checksum || (bytes > 0 && !src))
        return SPARROW_EINVAL;
    if (!al16(src) || !al4(checksum))
        return SPARROW_EINVAL;
    if (bytes == 0)
        return SPARROW_OK;
    return status_of(launch_stream_read(src, bytes, checksum, static_cast<hipStream_t>(stream)));
}

int32_t sparrow_budget_bound(const int32_t *seq_lens, int64_t num_seqs, int32_t page_size,
                             int32_t bin_tokens, int32_t n_bins, const int32_t *min_pages,
                             const int32_t *frac_num, int32_t frac_den, int32_t *budgets)
{
    if (num_seqs < 0 || page_size < 1 || bin_tokens < 1 || n_bins < 1 || frac_den < 1)
        return SPARROW_EINVAL;
    if (!min_pages || !frac_num || (num_seqs > 0 && !seq_lens))
        return SPARROW_EINVAL;
    for (int32_t i = 0; i < n_bins; ++i)
        if (min_pages[i] < 0 || frac_num[i] < 0)
            return SPARROW_EINVAL;
    const int64_t max_len = (int64_t)page_size * SPARROW_MAX_PAGES_PER_SEQ;
    int32_t best = 1;
    for (int64_t b = 0; b < num_seqs; ++b) {
        const int32_t L = seq_lens[b];
        if (L > max_len)
            return SPARROW_EINVAL;
        int32_t k = 0;
        if (L > 0) {
            const int bin = budget_bin(L, bin_tokens, n_bins);
            k = budget_from(L, page_size, min_pages[bin], frac_num[bin], frac_den, 0x7fffffff);
        }
        if (budgets)
            budgets[b] = k;
        if (k > best)
            best = k;
    }
    return best;
}

size_t sparrow_workspace_size(const sparrow_shape_t *shape, int32_t k_max, int32_t op)
{
    if (check_shape(shape) != SPARROW_OK)
        return 0;
    switch (op) {
    case SPARROW_OP_SCORE_TOPK: return shape->batch > kMaxBatch ? 0 : score_topk_workspace(*shape);
    case SPARROW_OP_SPARSE_ATTN:
        return k_max < 1 || k_max > SPARROW_MAX_PAGES_PER_SEQ || shape->batch > kMaxBatch
                   ? 0
                   : plan_attention(*shape).workspace_bytes;
    case SPARROW_OP_DENSE_ATTN:
        return shape->batch > kMaxBatch ? 0 : plan_attention(*shape).workspace_bytes;
    case SPARROW_OP_DECODE_STEP:
        return k_max < 1 || k_max > SPARROW_MAX_PAGES_PER_SEQ || shape->batch > kMaxBatch
                   ? 0
                   : decode_step_workspace(*shape);
    default: return 0;
    }
}

const char *sparrow_status_string(int32_t status)
{
    switch (status) {
    case SPARROW_OK: return "ok";
    case SPARROW_EINVAL: return "invalid argument (null pointer or bad size)";
    case SPARROW_EUNSUPPORTED: return "unsupported head_dim, page size, group size or dtype";
    case SPARROW_EWORKSPACE: return "workspace missing or too small";
    case SPARROW_EHIP: return "kernel launch failed";
    default: return "unknown status";
    }
}

}  // extern "C"
