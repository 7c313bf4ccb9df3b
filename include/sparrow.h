/*
 * sparrow.h - C ABI of the MI355X (gfx950) sparse-decode attention library.
 *
 * One decode step of one attention layer over a paged KV cache, as used by
 * sparse rollout in Sparrow (arXiv 2606.08446):
 *
 *   1. sparrow_page_meta_update   per-page key min/max metadata (the page
 *                                 landmark scored in Sec. 3.3 / Appendix C),
 *                                 or sparrow_append_kv: write the decoded token's
 *                                 K/V and update its page's metadata in O(1),
 *   2. sparrow_page_score_topk    page scores against the current query, the
 *                                 per-sequence page budget from the dynamic
 *                                 sparsity schedule (Sec. 3.2 Method box) and
 *                                 the block top-k page selection (Sec. 2,
 *                                 Appendix D: block top-k attention),
 *   3. sparrow_sparse_decode_attn softmax attention over the selected pages only
 *                                 (the "sparse, no scoring" term of the sparse
 *                                 cost model, Eq. sparse-cost),
 *   4. sparrow_dense_decode_attn  the dense paged decode it is measured against
 *                                 (Eq. dense-cost).
 *   sparrow_append_score_topk fuses the append into step 2, and
 *   sparrow_decode_step runs the append and steps 2 and 3 in one call.
 *
 * Around it stand sparrow_residual_norm (between two blocks of a layer), sparrow_qk_norm_rope (in front of
 * the cache), the 8-bit cache's calls (*_e4m3), sparrow_shared_prefix_decode_attn (dense attention for
 * the samples of one prompt) and sparrow_sample (the next token from the head's logits).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Every array argument is a DEVICE pointer owned by the caller.  The library
 *    allocates nothing, keeps no state between calls and never synchronises:
 *    each call only validates its host-visible arguments and enqueues kernels
 *    on `stream` (a hipStream_t passed as void*; NULL = the null stream).
 *  - Return value: SPARROW_OK (0) or a negative status (see below).  Nothing is
 *    enqueued when a negative status is returned.  Device contents are checked
 *    only where an index could leave a buffer: a block-table entry outside
 *    [0, num_phys_pages) marks an absent page - no kernel reads or writes that
 *    physical page; scoring sees zero metadata for it (score 0), attention
 *    leaves its tokens out, and an append to it writes nothing - and page
 *    indices, lengths and budgets are clamped to what the shape allows (a
 *    negative length is an empty sequence; one beyond max_pages_per_seq *
 *    page_size tokens counts as that many, and its token is not appended).
 *  - Inputs must not change while a call's kernels run (order other streams'
 *    writes before them): seq_lens and the block table are read more than once,
 *    and workgroups that saw different lengths would split the work differently
 *    and use workspace that none of them wrote.
 *  - bf16 tensors are IEEE bfloat16 bit patterns.  NaN inputs are not supported.
 *  - Alignment: q, k_cache, v_cache, meta, out and workspace start on a 16-byte
 *    boundary and the int32 arrays on a 4-byte boundary (any hipMalloc or PyTorch
 *    allocation is); a misaligned pointer is rejected with SPARROW_EINVAL.
 *  - Layouts (row-major, no padding):
 *      q            bf16  [batch][num_q_heads][head_dim]
 *      k_cache      bf16  [num_phys_pages][num_kv_heads][page_size][head_dim]
 *      v_cache      bf16  [num_phys_pages][num_kv_heads][page_size][head_dim]
 *      meta         bf16  [num_phys_pages][num_kv_heads][2][head_dim]
 *                         (row 0: channel-wise min, row 1: channel-wise max), or with
 *                         SPARROW_LANDMARK_MEAN fp32 [num_phys_pages][num_kv_heads][head_dim]
 *                         (channel-wise sum of the page's valid keys) - 512 B per
 *                         (page, head) either way
 *      block_table  int32 [batch][max_pages_per_seq]  logical -> physical page
 *      seq_lens     int32 [batch]  tokens of each sequence, including the token
 *                                  being decoded (0 allowed)
 *      idx          int32 [batch][num_kv_heads][k_max]  selected logical pages
 *      out          fp32 or bf16 [batch][num_q_heads][head_dim]
 *    Sequence b uses logical pages 0 .. ceil(seq_lens[b] / page_size) - 1; the
 *    rest of its block-table row may be read (the array must be whole) but its
 *    values never matter.  Query head j reads KV head
 *    j / G with G = num_q_heads / num_kv_heads (grouped-query attention).
 *  - Supported shapes: head_dim == 128; page_size in {16, 32, 64, 128};
 *    landmark in {SPARROW_LANDMARK_MINMAX, SPARROW_LANDMARK_MEAN};
 *    num_q_heads a multiple of num_kv_heads with G <= 16;
 *    1 <= max_pages_per_seq <= SPARROW_MAX_PAGES_PER_SEQ;
 *    batch * num_kv_heads <= 65535; batch <= SPARROW_MAX_BATCH for the
 *    scoring and attention entry points.
 */
#ifndef SPARROW_H
#define SPARROW_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPARROW_OK 0
#define SPARROW_EINVAL (-1)       /* null pointer, negative or inconsistent size      */
#define SPARROW_EUNSUPPORTED (-2) /* head_dim, page size, group size or dtype not supported */
#define SPARROW_EWORKSPACE (-3)   /* workspace missing or smaller than required       */
#define SPARROW_EHIP (-4)         /* a kernel launch failed                           */

#define SPARROW_MAX_PAGES_PER_SEQ 15360
#define SPARROW_MAX_BATCH 8192

#define SPARROW_OUT_F32 0
#define SPARROW_OUT_BF16 1

#define SPARROW_LANDMARK_MINMAX 0 /* per page: channel-wise min and max of the keys (bf16)  */
#define SPARROW_LANDMARK_MEAN 1   /* per page: channel-wise sum of the keys (fp32); scored
                                     as the mean key                                       */

#define SPARROW_LOGITS_F32 0
#define SPARROW_LOGITS_BF16 1

#define SPARROW_STREAM_F32 0
#define SPARROW_STREAM_BF16 1

#define SPARROW_OP_SCORE_TOPK 0
#define SPARROW_OP_SPARSE_ATTN 1
#define SPARROW_OP_DENSE_ATTN 2
#define SPARROW_OP_DECODE_STEP 3

/* Shape of one layer's decode batch (host struct, read during the call only).
   `landmark` selects the page metadata (SPARROW_LANDMARK_*; 0 = min/max), used by the
   metadata, append and scoring entry points and ignored by attention. */
typedef struct sparrow_shape {
    int32_t batch;
    int32_t num_q_heads;
    int32_t num_kv_heads;
    int32_t head_dim;
    int32_t page_size;
    int32_t max_pages_per_seq;
    int64_t num_phys_pages;
    int32_t landmark;
} sparrow_shape_t;

/*
 * Dynamic sparsity schedule (Sec. 3.2 Method box: the budget grows with the
 * current length so that the tail acceptance rate stays constant; lengths are
 * grouped into bins of 2K tokens in the paper).  Host struct whose two tables
 * are DEVICE arrays of n_bins int32.  For a sequence of L >= 1 tokens and
 * n = ceil(L / page_size) pages:
 *     bin = min((L - 1) / bin_tokens, n_bins - 1)
 *     k   = clamp(max(min_pages[bin], ceil(n * frac_num[bin] / frac_den)), 1, n)
 * and k = 0 for L = 0.  A fixed budget is min_pages = {P}, frac_num = {0}; a
 * fixed fraction is min_pages = {0}, frac_num = {num}, frac_den = den.  When
 * k == n every page is kept (Appendix F: attention is dense while the context
 * fits the budget).  Requires bin_tokens >= 1, n_bins >= 1, frac_den >= 1 and
 * non-negative table entries.
 *
 * sink_pages s and local_pages l (0 = pure top-k) force the logical pages
 * [0, s) (attention sinks) and [n - l, n) (the most recent pages) into the
 * selection ahead of every scored page, lower index first; the rest of the budget
 * k goes by score.  Both >= 0.
 */
typedef struct sparrow_schedule {
    int32_t bin_tokens;
    int32_t n_bins;
    const int32_t *min_pages;
    const int32_t *frac_num;
    int32_t frac_den;
    int32_t sink_pages;
    int32_t local_pages;
} sparrow_schedule_t;

/*
 * Per-page key metadata (Sec. 3.3 and Appendix C: landmark scores; the
 * landmark is the channel-wise min and max of the page's keys).
 *
 * For every sequence b and every logical page p that overlaps the token range
 * [first_pos[b], seq_lens[b]), and for every KV head h and channel i:
 *     meta[phys][h][0][i] = min over the valid tokens t of the page of K[t][i]
 *     meta[phys][h][1][i] = max over the same tokens
 * (SPARROW_LANDMARK_MEAN: meta[phys][h][i] = the fp32 sum of K[t][i] over the same
 * tokens, added in token order)
 * where phys = block_table[b][p] and the valid tokens of page p are
 * p*page_size .. min((p+1)*page_size, seq_lens[b]) - 1.  Values are copied
 * exactly (bf16 in, bf16 out); -0 orders below +0.  first_pos == NULL rebuilds
 * every page of every sequence.  A decode step that has just written token
 * L-1 passes first_pos[b] = L-1.  Entries of first_pos below 0 are treated as
 * 0; entries >= seq_lens[b] update nothing.
 *
 * Arguments: shape (host), k_cache (device, layout above), block_table,
 * seq_lens, first_pos (device [batch] or NULL), meta (device, written), stream.
 * Errors: SPARROW_EINVAL for a null shape/k_cache/block_table/seq_lens/meta or
 * a bad size; SPARROW_EUNSUPPORTED for head_dim/page_size; SPARROW_EHIP.
 */
int sparrow_page_meta_update(const sparrow_shape_t *shape, const void *k_cache,
                             const int32_t *block_table, const int32_t *seq_lens,
                             const int32_t *first_pos, void *meta, void *stream);

/*
 * Appending the token being decoded (the per-token landmark upkeep of Sec. 3.3:
 * the page metadata follows every generated key).
 *
 * seq_lens[b] counts the new token, which goes to position L - 1 = seq_lens[b] - 1:
 * logical page (L - 1) / page_size, slot (L - 1) % page_size.  For every KV head h:
 *     k_cache[phys][h][slot][:] = k_new[b][h][:],  v_cache[phys][h][slot][:] = v_new[b][h][:]
 * with phys = block_table[b][(L - 1) / page_size], and the page's metadata becomes the
 * channel-wise min/max of its old metadata and the new key (the key itself when the
 * slot is 0); with SPARROW_LANDMARK_MEAN its key sum plus the new key.  This equals
 * the metadata rebuilt from the page's L - page*page_size valid tokens
 * (sparrow_page_meta_update) provided the old metadata described the tokens before
 * L - 1.  Sequences with seq_lens[b] < 1 or seq_lens[b] > max_pages_per_seq *
 * page_size are left untouched.  Sequences must use distinct physical pages.
 *
 * Arguments: shape (host); k_new, v_new (device bf16 [batch][num_kv_heads][head_dim]);
 * k_cache, v_cache, meta (device, updated in place); block_table, seq_lens (device);
 * stream.
 * Errors: SPARROW_EINVAL (null or misaligned pointer, bad size), SPARROW_EUNSUPPORTED,
 * SPARROW_EHIP.
 */
int sparrow_append_kv(const sparrow_shape_t *shape, const void *k_new, const void *v_new,
                      void *k_cache, void *v_cache, const int32_t *block_table,
                      const int32_t *seq_lens, void *meta, void *stream);

/*
 * Page scoring and block top-k selection (Sec. 3.3: landmark scores and top-k
 * page picking; Sec. 3.2: the budget from the sparsity schedule).
 *
 * For every sequence b and KV head h, each logical page p < n_b is scored
 *     S_h(p) = sum over the G query heads j of head h of
 *              sum_i max(q[b][j][i] * mn_i(p), q[b][j][i] * mx_i(p))
 * (an upper bound of q_j . k_t over the tokens of the page), with fp32
 * arithmetic; with SPARROW_LANDMARK_MEAN, S_h(p) = sum_j q_j . (sum(p) / n_valid(p)),
 * the query group against the page's mean key.  k_b is the schedule's budget (see
 * sparrow_schedule_t), capped at k_max.  The k_b pages of largest S_h are kept, ties going to the lower
 * page index (-0 equals +0), and written in ascending page order to
 * out_idx[b][h][0 .. k_b); the rest of the row up to k_max is set to -1.
 * out_k[b] = k_b.  When k_b == n_b no page is scored and every page is kept.
 *
 * Arguments: shape (host); q, meta, block_table, seq_lens (device);
 * schedule (host struct with device tables); 1 <= k_max <= SPARROW_MAX_PAGES_PER_SEQ
 * (the row length of out_idx; callers pass at least the largest budget); out_k (device [batch]);
 * out_idx (device [batch][num_kv_heads][k_max]); workspace of at least
 * sparrow_workspace_size(shape, k_max, SPARROW_OP_SCORE_TOPK) bytes (device,
 * contents need not be initialised); stream.
 * Errors: SPARROW_EINVAL (null pointers, k_max out of range, bad schedule sizes or negative
 * forced-page counts), SPARROW_EUNSUPPORTED, SPARROW_EWORKSPACE, SPARROW_EHIP.
 */
int sparrow_page_score_topk(const sparrow_shape_t *shape, const void *q, const void *meta,
                            const int32_t *block_table, const int32_t *seq_lens,
                            const sparrow_schedule_t *schedule, int32_t k_max, int32_t *out_k,
                            int32_t *out_idx, void *workspace, size_t ws_bytes, void *stream);

/*
 * sparrow_append_kv followed by sparrow_page_score_topk, in one pass: the scoring
 * kernel's workgroup that owns a sequence's last page writes the new K/V rows and that
 * page's metadata and scores the page from the updated metadata, so no separate
 * metadata pass runs.  Results (caches, meta, out_k, out_idx) are identical to the two
 * calls in sequence.  Arguments are those of the two calls; the workspace is that of
 * SPARROW_OP_SCORE_TOPK.
 * Errors: as sparrow_page_score_topk, plus SPARROW_EINVAL for a null or misaligned
 * k_new, v_new, k_cache or v_cache.
 */
int sparrow_append_score_topk(const sparrow_shape_t *shape, const void *q, const void *k_new,
                              const void *v_new, void *k_cache, void *v_cache, void *meta,
                              const int32_t *block_table, const int32_t *seq_lens,
                              const sparrow_schedule_t *schedule, int32_t k_max, int32_t *out_k,
                              int32_t *out_idx, void *workspace, size_t ws_bytes, void *stream);

/*
 * Sparse decode attention over the selected pages (block-sparse attention,
 * Sec. 2; the attention term of Eq. sparse-cost).
 *
 * For every sequence b and query head j (KV head h = j / G) the token set T is
 * the valid tokens of the pages idx[b][h][0 .. min(k[b], k_max)); entries
 * outside [0, n_b) are skipped.  Then
 *     z_t = scale * (q[b][j] . K[t]),  w_t = exp(z_t - max z) / sum exp(z - max z)
 *     out[b][j] = sum_t w_t V[t]
 * computed with bf16 operands and fp32 accumulation (the softmax weights are
 * rounded to bf16 before they multiply V).  An empty token set gives a zero
 * row.  out_dtype is SPARROW_OUT_F32 or SPARROW_OUT_BF16.
 * The order of the fp32 sums depends only on the shape, k_max, the page lists
 * and the device (its count of resident waves), so repeated calls on one GPU
 * give identical results.  A call with at most 256
 * (sequence, KV head) units, at most 8 query heads per KV head,
 * k_max * page_size <= 1024 and max_pages_per_seq <= 4096 runs one workgroup
 * per unit and leaves the workspace untouched; larger calls split the lists
 * over all resident waves and merge partials kept in the workspace.  With every page listed and k_max
 * equal to max_pages_per_seq the result equals sparrow_dense_decode_attn's bit
 * for bit (the dense call's list bound is max_pages_per_seq).
 *
 * Arguments: shape (host); q, k_cache, v_cache, block_table, seq_lens, k
 * (device [batch]), idx (device [batch][num_kv_heads][k_max]);
 * 1 <= k_max <= SPARROW_MAX_PAGES_PER_SEQ;
 * scale (typically 1/sqrt(head_dim)); out (device, written); out_dtype;
 * workspace of at least sparrow_workspace_size(shape, k_max,
 * SPARROW_OP_SPARSE_ATTN) bytes; stream.
 * Errors: SPARROW_EINVAL, SPARROW_EUNSUPPORTED, SPARROW_EWORKSPACE, SPARROW_EHIP.
 */
int sparrow_sparse_decode_attn(const sparrow_shape_t *shape, const void *q, const void *k_cache,
                               const void *v_cache, const int32_t *block_table,
                               const int32_t *seq_lens, const int32_t *k, const int32_t *idx,
                               int32_t k_max, float scale, void *out, int32_t out_dtype,
                               void *workspace, size_t ws_bytes, void *stream);

/*
 * sparrow_sparse_decode_attn for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation): the same
 * computation and results, with the workspace taken from a buffer of
 * SPARROW_NOALLOC_SCRATCH_BYTES that the library holds on each GPU it runs on (from the
 * first call on that GPU until the process ends).  The call allocates nothing.
 *
 * Every call on one GPU uses that GPU's buffer: calls that can overlap on one GPU (on
 * different streams, or from several host threads without ordering) race and must not be
 * issued; calls in one stream are ordered and safe.  The buffer needs no initialisation.
 * Shapes whose workspace (sparrow_workspace_size with SPARROW_OP_SPARSE_ATTN) exceeds
 * SPARROW_NOALLOC_SCRATCH_BYTES are refused with SPARROW_EWORKSPACE; the Qwen3-shaped decode
 * batches here need 5-13 MiB.
 *
 * Arguments and the other errors are those of sparrow_sparse_decode_attn without the
 * workspace; SPARROW_EHIP also when the buffer's address cannot be obtained.
 */
#define SPARROW_NOALLOC_SCRATCH_BYTES 33554432 /* 32 MiB */
int sparrow_sparse_decode_attn_noalloc(const sparrow_shape_t *shape, const void *q,
                                       const void *k_cache, const void *v_cache,
                                       const int32_t *block_table, const int32_t *seq_lens,
                                       const int32_t *k, const int32_t *idx, int32_t k_max,
                                       float scale, void *out, int32_t out_dtype, void *stream);

/*
 * One decode step of one layer in one call (the whole sparse step of Sec. 3.3:
 * append, landmark scores, the schedule's budget of Sec. 3.2, block top-k and
 * attention over the selected pages): sparrow_append_score_topk - or
 * sparrow_page_score_topk when k_new and v_new are both NULL - followed by
 * sparrow_sparse_decode_attn on the selection it made (k = out_k, idx =
 * out_idx).  Results (caches, meta, out_k, out_idx, out) equal those of the two
 * calls in sequence bit for bit.  When the attention call would run one
 * workgroup per unit (see sparrow_sparse_decode_attn), the selection stays on
 * chip: the whole step is one kernel, or behind a wide block table the scoring
 * kernel and one for the budget, the top-k and the attention.
 *
 * Arguments: those of the two calls (k_new and v_new both NULL or both set);
 * workspace of at least sparrow_workspace_size(shape, k_max,
 * SPARROW_OP_DECODE_STEP) bytes.
 * Errors: those of the two calls.
 */
int sparrow_decode_step(const sparrow_shape_t *shape, const void *q, const void *k_new,
                        const void *v_new, void *k_cache, void *v_cache, void *meta,
                        const int32_t *block_table, const int32_t *seq_lens,
                        const sparrow_schedule_t *schedule, int32_t k_max, float scale,
                        int32_t *out_k, int32_t *out_idx, void *out, int32_t out_dtype,
                        void *workspace, size_t ws_bytes, void *stream);

/*
 * Dense paged decode attention (the dense rollout baseline, Eq. dense-cost):
 * the same as sparrow_sparse_decode_attn with T = every valid token of the
 * sequence, and max_pages_per_seq in place of k_max when choosing between one
 * workgroup per unit and the streaming split.
 *
 * Arguments as above, without k/idx/k_max; workspace of at least
 * sparrow_workspace_size(shape, 0, SPARROW_OP_DENSE_ATTN) bytes.
 * Errors: SPARROW_EINVAL, SPARROW_EUNSUPPORTED, SPARROW_EWORKSPACE, SPARROW_EHIP.
 */
int sparrow_dense_decode_attn(const sparrow_shape_t *shape, const void *q, const void *k_cache,
                              const void *v_cache, const int32_t *block_table,
                              const int32_t *seq_lens, float scale, void *out, int32_t out_dtype,
                              void *workspace, size_t ws_bytes, void *stream);

/*
 * Dense decode attention for sequences in groups whose first tokens are the same - the samples of one
 * prompt - with the shared pages read once per group instead of once per sequence.
 *
 * Group g holds the sequences cu_groups[g] .. cu_groups[g+1] - 1 and shares the s = prefix_lens[g] /
 * page_size whole pages (rounded down) at the start of its sequences: token t < s * page_size of each is read
 * from the pages that the block-table row of the group's FIRST sequence lists, whatever that
 * sequence's own length; the sequences' other tokens from their own rows, whose first s entries are
 * not read.  (A prompt that ends inside a page leaves its last tokens in every sequence's own copy of
 * that page.)  A sequence shorter than the prefix attends to its own seq_lens[b] tokens of it.
 * Groups of one sequence, and sequences in no group, share nothing.  With that the result is
 * sparrow_dense_decode_attn's,
 *     out[b][j] = sum_t w_t V[t],  w = softmax(scale * q[b][j] . K[t]) over t < seq_lens[b]
 * with fp32 sums and fp32 softmax numerators (all of their 24 bits enter the product with V), rounded once
 * for SPARROW_OUT_BF16.  An empty sequence gives a zero row.  The order of the
 * sums depends only on the shape, the groups, the lengths and the device.  What lies behind a
 * sequence's end may hold anything, the shared tokens that only longer sequences of its group reach too.
 *
 * Arguments: as for sparrow_dense_decode_attn, batch * num_kv_heads <= 65535; 0 <= num_groups <=
 * SPARROW_MAX_GROUPS; cu_groups (device int32 [num_groups + 1], non-decreasing; entries outside [0,
 * batch] count as the nearer end, one below an earlier entry as that one), prefix_lens (device int32
 * [num_groups]; what the block table cannot hold, or is negative, counts as the nearer end), both
 * NULL allowed without groups; scale finite; workspace of at least
 * sparrow_shared_prefix_workspace_size(shape, num_groups) bytes.
 * Errors: SPARROW_EINVAL, SPARROW_EUNSUPPORTED, SPARROW_EWORKSPACE, SPARROW_EHIP.
 */
#define SPARROW_MAX_GROUPS 4096
int sparrow_shared_prefix_decode_attn(const sparrow_shape_t *shape, const void *q,
                                      const void *k_cache, const void *v_cache,
                                      const int32_t *block_table, const int32_t *seq_lens,
                                      int32_t num_groups, const int32_t *cu_groups,
                                      const int32_t *prefix_lens, float scale, void *out,
                                      int32_t out_dtype, void *workspace, size_t ws_bytes,
                                      void *stream);

/* Workspace bytes of sparrow_shared_prefix_decode_attn; 0 for a shape that it refuses. */
size_t sparrow_shared_prefix_workspace_size(const sparrow_shape_t *shape, int32_t num_groups);

/*
 * Per-token acceptance rate between the dense policy and the sparse rollout
 * (Sec. 3.1, Eq. 1: the expectation under the draft of min(p/q, 1), which equals
 * the sum over the vocabulary of min(p(x), q(x))).
 *
 * For every token t < num_tokens, with a = target_logits[t][:] (dense policy) and
 * b = draft_logits[t][:] (sparse rollout), rows of `vocab` entries:
 *     p = softmax(inv_temperature * a),  q = softmax(inv_temperature * b),
 *     alpha[t] = sum_x min(p(x), q(x))
 * computed in fp32 (two passes: log-sum-exp of both rows, then the sum).  Agrees
 * with an fp64 evaluation to about 1e-5.  A logit of -inf (a masked vocabulary entry)
 * has probability 0; each row needs at least one finite logit, and -inf entries need
 * inv_temperature > 0.  NaN and +inf logits are not supported.  logits_dtype is SPARROW_LOGITS_F32 or
 * SPARROW_LOGITS_BF16; rows are contiguous ([num_tokens][vocab], row-major).
 *
 * Arguments: num_tokens >= 0; vocab >= 1; target_logits, draft_logits (device,
 * element-aligned); inv_temperature finite; alpha (device fp32 [num_tokens],
 * written); stream.
 * Errors: SPARROW_EINVAL (null/misaligned pointer, bad size, non-finite
 * temperature), SPARROW_EUNSUPPORTED (dtype), SPARROW_EHIP.
 */
int sparrow_acceptance_rate(int64_t num_tokens, int32_t vocab, int32_t logits_dtype,
                            const void *target_logits, const void *draft_logits,
                            float inv_temperature, float *alpha, void *stream);

/*
 * The approximation of the paper's measurement (Sec. 3.1, footnote: the inference
 * engine returns the top-20 tokens and their log-probabilities per position):
 *     alpha[t] = sum_{i < k} min(exp(lp_target[t][i]), exp(lp_draft[t][i]))
 * over the k listed tokens, whose normalised log-probabilities under the two
 * distributions are given (fp32 [num_tokens][k], device).  A lower bound of the
 * exact rate.
 * Errors: SPARROW_EINVAL (null/misaligned pointer, num_tokens < 0, k < 1), SPARROW_EHIP.
 */
int sparrow_acceptance_rate_topk(int64_t num_tokens, int32_t k, const float *lp_target,
                                 const float *lp_draft, float *alpha, void *stream);

/*
 * The next token of every row of logits, drawn with a given random number.
 *
 * For every row t < num_rows, z = logits[t][:], T = temperature[t], m = max z, x_i = (z_i - m) / T,
 * w_i = exp(x_i), tokens ordered by z descending, equal ones by index ascending (-0 equals +0):
 *     top-k   (1 <= top_k[t] < vocab)  keeps the first top_k[t] tokens of that order;
 *     top-p   (top_p[t] < 1)   keeps of these each one whose predecessors' w add up to less than
 *                              top_p[t] times the sum of w over all of these, the first one always;
 *     min-p   (min_p[t] > 0)   keeps of these those with w_i >= min(min_p[t], 1).
 *     tokens[t]   = the first kept token, by index, at which the running sum of the kept w exceeds
 *                   uniform[t] times their whole sum
 *     logprobs[t] = log of its w over that sum: the log-probability that it was drawn with
 * Other values of top_k, top_p and min_p leave a filter off, as NULL arrays do; temperature NULL is 1.
 * T <= 0 (or NaN) takes the largest logit, the lowest index of equal ones, with logprobs[t] = 0; so do
 * top_k[t] == 1 and top_p[t] <= 0.  uniform[t] is clamped to [0, 1 - 2^-24].  -inf and NaN logits are
 * masked tokens, never drawn; +inf counts as the largest finite number.  A row with no other gets
 * tokens[t] = -1 and logprobs[t] = -inf.  Weights and their sums are held to 1e-13 of the sum, so that
 * the token is the definition's unless a border lies closer; results do not depend on the launch.
 *
 * Arguments: 0 <= num_rows < 2^31; 1 <= vocab <= SPARROW_SAMPLE_MAX_VOCAB; logits_dtype
 * (SPARROW_LOGITS_*); logits (device, element-aligned, rows of row_stride >= vocab elements: any
 * stride); temperature, top_p, min_p (device fp32 [num_rows] or NULL), top_k (device int32 [num_rows]
 * or NULL); uniform (device fp32 [num_rows]); tokens (device int32 [num_rows], written); logprobs
 * (device fp32 [num_rows], written, or NULL); workspace of at least sparrow_sample_workspace_size
 * bytes (device, 16-byte aligned, scratch of this call: calls that may overlap need one each); stream.
 * Errors: SPARROW_EINVAL, SPARROW_EUNSUPPORTED (vocab, dtype), SPARROW_EWORKSPACE, SPARROW_EHIP.
 */
#define SPARROW_SAMPLE_MAX_VOCAB 524288
int sparrow_sample(int64_t num_rows, int32_t vocab, int32_t logits_dtype, const void *logits,
                   int64_t row_stride, const float *temperature, const int32_t *top_k,
                   const float *top_p, const float *min_p, const float *uniform, int32_t *tokens,
                   float *logprobs, void *workspace, size_t ws_bytes, void *stream);

/* Workspace bytes of sparrow_sample; 0 for sizes that it refuses (and for no rows). */
size_t sparrow_sample_workspace_size(int64_t num_rows, int32_t vocab, int32_t logits_dtype);

/*
 * Lower-tail statistic of the acceptance rate per length bin (Sec. 3.1 Method:
 * the 5-percentile of the per-token rate; Sec. 3.2: tokens grouped by position
 * in 2K-token bins).
 *
 * Token t (alpha[t], positions[t]) belongs to bin min(positions[t] / bin_tokens,
 * n_bins - 1); tokens with a negative position are ignored.  For each bin b:
 * count[b] = its number of tokens N, mean[b] = the fp64 mean of their alpha, and
 * quantile[b] = the `percentile`-percentile with linear interpolation between
 * order statistics: with the values sorted x_0 <= ... <= x_{N-1},
 * h = (N - 1) * percentile / 100, lo = floor(h),
 * quantile = x_lo + (h - lo) * (x_{lo+1} - x_lo)   (x_lo when lo = N - 1),
 * in fp64.  Empty bins get count 0 and NaN mean and quantile.
 *
 * Arguments: num_tokens >= 0; alpha (device fp32), positions (device int32), both
 * may be NULL when num_tokens is 0;
 * bin_tokens >= 1; 1 <= n_bins <= 65535; 0 <= percentile <= 100; quantile,
 * mean (device fp64 [n_bins]) and count (device int64 [n_bins]), written; stream.
 * Errors: SPARROW_EINVAL, SPARROW_EHIP.
 */
int sparrow_tail_stats(int64_t num_tokens, const float *alpha, const int32_t *positions,
                       int32_t bin_tokens, int32_t n_bins, double percentile, double *quantile,
                       double *mean, int64_t *count, void *stream);

/*
 * RMS norm of every query and key head and the position rotation, in one pass: what stands
 * between a layer's projections and the decode step (the workloads' models normalise each head).
 *
 * For every token t < num_tokens with positions[t] >= 0, every head j of q (num_q_heads of them,
 * weight w = q_weight) and of k (num_k_heads, w = k_weight), with x its row of 128 channels:
 *     r = 1 / sqrt(mean(x^2) + eps),  n_i = x_i r w_i,  a_i = positions[t] * inv_freq[i]
 *     y_i = n_i cos a_i - n_{i+64} sin a_i,  y_{i+64} = n_{i+64} cos a_i + n_i sin a_i   (i < 64)
 * written to q_out, k_out.  fp32 arithmetic (the angle in fp64), one rounding to bf16.  Rows of a
 * token with a negative position (padding) are left as they were.  inv_freq holds any
 * frequencies, in radians per token, scaled ones included.  The sum of squares is fp32: rows with
 * entries beyond 1e18 overflow it, and with eps = 0 a row of zeros, or of entries below 1e-19, has no
 * finite 1 / sqrt.
 *
 * Arguments: 0 <= num_tokens < 2^31; 1 <= num_q_heads, num_k_heads <= 1024; head_dim == 128; q, k
 * (device bf16, 16-byte aligned; head j of token t starts at t * stride + j * 128 elements; the strides
 * are multiples of 8 and at least num_heads * 128, so that both may lie in one fused projection
 * output); q_weight, k_weight (device bf16 [128], 16-byte aligned); inv_freq (device fp64 [64], 8-byte
 * aligned); positions (device int32 [num_tokens]); eps >= 0; q_out, k_out (device bf16
 * [num_tokens][num_heads][128], written, 16-byte aligned; either may be its input where that is
 * contiguous); stream.
 * Errors: SPARROW_EINVAL, SPARROW_EUNSUPPORTED (head_dim), SPARROW_EHIP.
 */
int sparrow_qk_norm_rope(int64_t num_tokens, int32_t num_q_heads, int32_t num_k_heads,
                         int32_t head_dim, const void *q, int64_t q_stride, const void *k,
                         int64_t k_stride, const void *q_weight, const void *k_weight,
                         const double *inv_freq, const int32_t *positions, float eps,
                         void *q_out, void *k_out, void *stream);

/*
 * Gradient of sparrow_qk_norm_rope.  With dy a row of dq_out or dk_out and g its rotation by the
 * negative angle, u_i = g_i w_i:
 *     dx_i = r (u_i - x_i r mean(u x r)),   dw_i = sum over tokens and heads of g_i x_i r
 * dx goes to dq, dk (bf16, strided like q and k, so that both may lie in one buffer; either may
 * be the array it derives from, with the same strides), dw to dq_weight, dk_weight (fp32 [128]
 * each, overwritten; fp32 sums in an order that depends on the sizes alone).  Tokens with a
 * negative position get dx = 0 and add nothing to dw.
 *
 * Arguments: as above; dq_out, dk_out (device bf16 [num_tokens][num_heads][128]); workspace of at
 * least SPARROW_ROPE_WORKSPACE_BYTES (device, 16-byte aligned, scratch of this call: calls that may
 * overlap need one each); stream.
 * Errors: as above, plus SPARROW_EWORKSPACE.
 */
#define SPARROW_ROPE_WORKSPACE_BYTES 1048576
int sparrow_qk_norm_rope_bwd(int64_t num_tokens, int32_t num_q_heads, int32_t num_k_heads,
                             int32_t head_dim, const void *dq_out, const void *dk_out,
                             const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                             const void *q_weight, const void *k_weight, const double *inv_freq,
                             const int32_t *positions, float eps, void *dq, int64_t dq_stride,
                             void *dk, int64_t dk_stride, float *dq_weight, float *dk_weight,
                             void *workspace, size_t ws_bytes, void *stream);

/*
 * The residual stream after a block and the norm before the next one, in one pass: what stands between
 * two blocks of a layer, for models with a norm on one side of a block or on both, a gate and a
 * residual scale.
 *
 * For every token t < num_tokens, with rows of `channels` values:
 *     n = x r_x post_weight,  r_x = 1 / sqrt(mean(x^2) + eps)      (post_weight NULL: n = x)
 *     h' = h + scale * sigmoid(gate) * n                           (gate NULL: h + scale * n)
 *     y = h' r weight,  r = 1 / sqrt(mean(h'^2) + eps)
 * h' goes to h_out in the stream's type and y to y, each rounded once from fp32 (y comes from h' as
 * it is before that rounding).  With x == NULL there is no block yet: y = h r weight, and gate,
 * post_weight and h_out are NULL too.  The sums of squares are fp32: entries beyond 1e18 overflow
 * them, and with eps = 0 a row of zeros, or of entries below 1e-19, has no finite 1 / sqrt.
 *
 * Arguments: 0 <= num_tokens < 2^31; channels a multiple of 8, at most 16384; stream_dtype
 * (SPARROW_STREAM_*: the type of h and h_out); h (device [num_tokens][channels]); x, gate (device
 * bf16, rows of x_stride and gate_stride elements, multiples of 8 and at least channels, so that
 * both may lie in one projection's output); weight, post_weight (device bf16 [channels]); scale
 * finite; eps >= 0; h_out (device, like h, written; may be h); y (device bf16
 * [num_tokens][channels], written); all 16-byte aligned; stream.
 * Errors: SPARROW_EINVAL, SPARROW_EUNSUPPORTED (channels, stream_dtype), SPARROW_EHIP.
 */
int sparrow_residual_norm(int64_t num_tokens, int32_t channels, int32_t stream_dtype, const void *h,
                          const void *x, int64_t x_stride, const void *gate, int64_t gate_stride,
                          const void *weight, const void *post_weight, float scale, float eps,
                          void *h_out, void *y, void *stream);

/*
 * Gradient of sparrow_residual_norm, from the stream behind the block (h_out, as it was written).
 * With dy the gradient of y, dh_out that of h_out from everything behind (NULL: zero), u = dy weight,
 * k = h_out r, s = sigmoid(gate):
 *     dh = dh_out + r (u - k mean(u k)),              dweight = sum over the tokens of dy k
 *     d = scale dh,  e = d s,  dgate = d n s (1 - s)  (without a gate e = d)
 *     dx = r_x (v - k_x mean(v k_x)),  v = e post_weight,  k_x = x r_x,  dpost_weight = sum of e k_x
 *     (without post_weight dx = e)
 * fp32 arithmetic; dh is rounded to the stream's type, dx and dgate to bf16; dweight and dpost_weight
 * are fp32 [channels], overwritten, summed in an order that depends on the sizes alone.
 *
 * Arguments: as above; dy (device bf16 [num_tokens][channels]); dh_out (like h_out, or NULL); x may
 * be NULL where neither gate nor post_weight is given; dh (like h_out, written; may be dh_out); dx,
 * dgate (device bf16 rows of dx_stride and dgate_stride elements, written; dx NULL: there is no
 * block; dgate NULL exactly where gate is); dweight; dpost_weight (NULL exactly where post_weight is);
 * workspace of at least sparrow_residual_norm_workspace_size(num_tokens, channels) bytes (device,
 * 16-byte aligned, scratch of this call: calls that may overlap need one each); stream.  With
 * num_tokens == 0 nothing is written.
 * Errors: as above, plus SPARROW_EWORKSPACE.
 */
int sparrow_residual_norm_bwd(int64_t num_tokens, int32_t channels, int32_t stream_dtype,
                              const void *dy, const void *dh_out, const void *h_out, const void *x,
                              int64_t x_stride, const void *gate, int64_t gate_stride,
                              const void *weight, const void *post_weight, float scale, float eps,
                              void *dh, void *dx, int64_t dx_stride, void *dgate,
                              int64_t dgate_stride, float *dweight, float *dpost_weight,
                              void *workspace, size_t ws_bytes, void *stream);

/* Workspace bytes of sparrow_residual_norm_bwd; 0 for sizes that it refuses (and for no tokens). */
size_t sparrow_residual_norm_workspace_size(int64_t num_tokens, int32_t channels);

/*
 * The e4m3 cache: K and V in 8 bits, half the bytes that a decode step streams.
 *
 *     k_cache, v_cache  e4m3  [num_phys_pages][num_kv_heads][page_size][128]   (OCP float8 e4m3,
 *                             no infinities)
 *     exps              uint8 [num_phys_pages][num_kv_heads][page_size / 4][2][4]: for every four
 *                             tokens K's four bytes, then V's
 * A channel of a row of K (V) is code * 2^(byte - 127) with the row's byte of K (V).  From a bf16
 * row with largest magnitude m, byte - 127 is the least integer e with m <= 448 * 2^e, clamped to
 * [-117, 119], and code = x * 2^-e rounded to nearest even (clamped to +-448, which only a row
 * beyond 448 * 2^119 reaches).  The scale is a power of two, so every value is exactly a bf16 number:
 * what sparrow_read_kv_e4m3 returns is what the cache holds, and the bf16 entry points applied to
 * it describe the 8-bit ones.
 *
 * sparrow_append_kv_e4m3 writes new tokens.  Sequence b's rows are cu_tokens[b] .. cu_tokens[b+1] - 1
 * (n_b of them); they go to the positions seq_lens[b] - n_b .. seq_lens[b] - 1, and seq_lens counts
 * them.  With cu_tokens == NULL every sequence has one row (num_tokens == batch): the decode step.
 * The landmarks of the pages that they land on follow, from the values as the cache holds them: for
 * a page whose slot 0 is among the new tokens they are its new tokens' min/max (or fp32 sum in
 * token order), else the old landmarks joined with them - what sparrow_page_meta_update would make
 * of the cache's values.  Selection (sparrow_page_score_topk) then works on meta as ever.  A
 * sequence with seq_lens[b] < 1 or > max_pages_per_seq * page_size is left untouched, tokens before
 * position 0 and on absent pages are dropped, and rows behind cu_tokens[batch] are not read.
 * cu_tokens is non-decreasing; entries outside [0, num_tokens] count as the nearer end.  Sequences
 * must use distinct physical pages.  NaN is not supported; an infinity becomes 448 * 2^119.
 *
 * Arguments: shape (host); k_new, v_new (device bf16: head h of row r starts at r * stride + h * 128
 * elements; strides are multiples of 8 and at least num_kv_heads * 128); cu_tokens (device int32
 * [batch + 1], or NULL); 0 <= num_tokens <= 134217728 (rows that k_new and v_new have); k_cache,
 * v_cache, exps (device; caches on 16, exps on 8 bytes; updated in place); block_table, seq_lens
 * (device); meta (device, updated); stream.
 * Errors: SPARROW_EINVAL, SPARROW_EUNSUPPORTED, SPARROW_EHIP.
 */
int sparrow_append_kv_e4m3(const sparrow_shape_t *shape, const void *k_new, int64_t k_stride,
                           const void *v_new, int64_t v_stride, const int32_t *cu_tokens,
                           int64_t num_tokens, void *k_cache, void *v_cache, void *exps,
                           const int32_t *block_table, const int32_t *seq_lens, void *meta,
                           void *stream);

/*
 * The last n_b = cu_tokens[b+1] - cu_tokens[b] tokens of every sequence from an e4m3 cache, as bf16
 * rows cu_tokens[b] .. of k_out and v_out [num_tokens][num_kv_heads][128] (exact).  Rows of positions
 * before 0, past the block table or on absent pages are zeros; rows behind cu_tokens[batch] are left
 * as they were.  cu_tokens as above (NULL: the last token of each).
 *
 * Errors: as above.
 */
int sparrow_read_kv_e4m3(const sparrow_shape_t *shape, const void *k_cache, const void *v_cache,
                         const void *exps, const int32_t *block_table, const int32_t *seq_lens,
                         const int32_t *cu_tokens, int64_t num_tokens, void *k_out, void *v_out,
                         void *stream);

/*
 * Decode attention of one new token per sequence over an e4m3 cache: sparrow_sparse_decode_attn and
 * sparrow_dense_decode_attn with K and V as the cache's values,
 *     z_t = scale * 2^(kbyte_t - 127) * (q[b][j] . kcode_t),  w = softmax(z),
 *     out[b][j] = sum_t w_t 2^(vbyte_t - 127) vcode_t
 * with fp32 sums and fp32 softmax numerators (all of their 24 bits enter the product with V).  Page lists, lengths, absent pages and empty sequences are those calls'; so is the
 * workspace (SPARROW_OP_SPARSE_ATTN, SPARROW_OP_DENSE_ATTN).  The order of the sums depends only on the
 * shape, k_max, the page lists and the device.
 *
 * Arguments: as there, with k_cache, v_cache (16-byte aligned) and exps (8-byte aligned) of an e4m3
 * cache of num_phys_pages * num_kv_heads * page_size / 16 < 2^31.
 * Errors: SPARROW_EINVAL, SPARROW_EUNSUPPORTED, SPARROW_EWORKSPACE, SPARROW_EHIP.
 */
int sparrow_sparse_decode_attn_e4m3(const sparrow_shape_t *shape, const void *q,
                                    const void *k_cache, const void *v_cache, const void *exps,
                                    const int32_t *block_table, const int32_t *seq_lens,
                                    const int32_t *k, const int32_t *idx, int32_t k_max,
                                    float scale, void *out, int32_t out_dtype, void *workspace,
                                    size_t ws_bytes, void *stream);
int sparrow_dense_decode_attn_e4m3(const sparrow_shape_t *shape, const void *q,
                                   const void *k_cache, const void *v_cache, const void *exps,
                                   const int32_t *block_table, const int32_t *seq_lens,
                                   float scale, void *out, int32_t out_dtype, void *workspace,
                                   size_t ws_bytes, void *stream);

/*
 * Read-only streaming reference (a measurement helper, not a step of the method): reads
 * `bytes` bytes at src once, with the 16-byte non-temporal vector loads and the
 * consecutive-lanes layout of the decode-step kernels, from a grid that keeps every
 * compute unit busy, and adds every 32-bit word of the buffer into *checksum (modulo
 * 2^32, on top of its current value: the caller sets it, usually to 0).  Timing a call
 * gives the rate a pure read stream sustains on the device, the practical ceiling of the
 * read-dominated decode kernels beside the HBM peak.
 *
 * Arguments: src (device, 16-byte aligned, may be NULL when bytes is 0); bytes >= 0, a
 * multiple of 16; checksum (device uint32, 4-byte aligned); stream.
 * Errors: SPARROW_EINVAL (null or misaligned pointer, bad size), SPARROW_EHIP.
 */
int sparrow_stream_read(const void *src, int64_t bytes, uint32_t *checksum, void *stream);

/*
 * Host-side page budgets of the dynamic sparsity schedule (Sec. 3.2 Method box; the
 * formula of sparrow_schedule_t, evaluated by the same code the scoring kernels use), to
 * size k_max before a call of sparrow_page_score_topk or sparrow_append_score_topk.
 *
 * For every b < num_seqs: budgets[b] = k_b of a sequence of seq_lens[b] tokens (0 when
 * seq_lens[b] <= 0), not capped by any k_max.  Returns max(1, max_b k_b), the smallest
 * k_max that caps no budget, or a negative status.
 *
 * Arguments: seq_lens (HOST int32 [num_seqs], may be NULL when num_seqs is 0); num_seqs
 * >= 0; page_size >= 1; bin_tokens >= 1; n_bins >= 1; min_pages, frac_num (HOST int32
 * [n_bins], non-negative); frac_den >= 1; budgets (HOST int32 [num_seqs], written) or
 * NULL.  Every pointer is a host pointer; nothing runs on the GPU.
 * Errors: SPARROW_EINVAL (bad size, null table, negative table entry, or a length above
 * page_size * SPARROW_MAX_PAGES_PER_SEQ).
 */
int32_t sparrow_budget_bound(const int32_t *seq_lens, int64_t num_seqs, int32_t page_size,
                             int32_t bin_tokens, int32_t n_bins, const int32_t *min_pages,
                             const int32_t *frac_num, int32_t frac_den, int32_t *budgets);

/*
 * Workspace bytes needed by one call of `op` (SPARROW_OP_*: SCORE_TOPK for the
 * two scoring calls, SPARSE_ATTN, DENSE_ATTN, DECODE_STEP) with this shape
 * and k_max (ignored for SPARROW_OP_DENSE_ATTN).  Returns 0 for an invalid or
 * unsupported shape.  The workspace holds scratch results of one call only;
 * calls that run concurrently need separate workspaces.
 */
size_t sparrow_workspace_size(const sparrow_shape_t *shape, int32_t k_max, int32_t op);

/* Static, human-readable name of a status code. */
const char *sparrow_status_string(int32_t status);

#ifdef __cplusplus
}
#endif

#endif /* SPARROW_H */
