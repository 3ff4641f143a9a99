/* Operators of libppd for programs that run a model's layers themselves, beside ppd_early_topk (ppd.h): the keys and
 * values of many sequences in pages, the attention of new tokens over them, and the verification of drafted tokens
 * against the target model's logits.  Together they make a step that checks drafts: the last token and the drafts of
 * every sequence go through the layers as one ragged batch (ppd_paged_append and ppd_paged_attention in each), and
 * ppd_verify_drafts turns the logits of all their rows into the tokens to emit.  What a rejected draft left in the
 * pages needs no undoing: the next step's tokens are written over it.
 *
 * All three only queue their work on hip_stream (a hipStream_t of the current device, NULL = its default stream): they
 * allocate nothing, wait for nothing, keep nothing from call to call but a count of attention's (the number that a call's
 * workgroups mark their scratch memory with), and may be captured into HIP graphs.  Tensors are DEVICE memory, borrowed
 * until the queued work has run; the structs are HOST and are read before the call returns.
 * Scratch memory is the caller's; calls whose work may overlap in time need scratch of their own each, and so do graphs
 * whose replays may overlap.
 * Return codes as in ppd.h: PPD_EINVAL before anything is queued, PPD_ELIMIT for sizes beyond a stated maximum,
 * PPD_EHIP if a launch failed (ppd_last_hip_error(NULL)).  What lies in DEVICE memory (lengths, page numbers, token ids)
 * cannot be checked by the host: the kernels check it, and what would lie outside a tensor is neither read nor written. */
#ifndef PPD_LAYERS_H
#define PPD_LAYERS_H
#include "ppd.h"
#ifdef __cplusplus
extern "C" {
#endif

#define PPD_FP32 0
#define PPD_BF16 1
#define PPD_FP16 2

#define PPD_MAX_SEQS 4096
#define PPD_MAX_TOKENS (1 << 22)
#define PPD_MAX_HEADS 1024

/* Keys and values in pages: k and v are [n_pages][page_size][n_kv_heads][head_dim], in any order of the first three
 * that the strides (in elements) express; head_dim is contiguous (strides of 0: for ppd_paged_attention only).  Every row of head_dim elements begins at a multiple
 * of 16 bytes (so do the tensors, and so do all strides). */
typedef struct {
  void *k, *v;
  int64_t k_page, k_pos, k_head;
  int64_t v_page, v_pos, v_head;
  int32_t n_pages;
  int32_t page_size;  /* positions of a page, at least 1 */
  int32_t n_kv_heads;
  int32_t head_dim;   /* 64 or 128 */
  int32_t dtype;      /* PPD_FP32, PPD_BF16, PPD_FP16: of the pages and of every row of queries, keys, values and outputs */
} ppd_paged_cache;

/* A ragged batch of new tokens.  Sequence s has rows q_start[s] .. q_start[s+1]-1 (none: it takes no part), which are its
 * last tokens: of its kv_len[s] positions, new tokens included, row q_start[s] + i is at position
 * kv_len[s] - (q_start[s+1] - q_start[s]) + i.  Position p lies in slot p % page_size of page
 * pages[s * pages_stride + p / page_size].  A page number outside [0, n_pages) (-1, say) and a place behind max_pages
 * mean that there is no page: such positions are not written by ppd_paged_append and not seen by ppd_paged_attention.
 * Rows behind the last sequence (q_start[n_seqs] < n_tokens, a padded batch) and before the first are not touched.
 * q_start must not decrease (if it does, which rows of the outputs are written, and what to them, is undefined).  All three
 * arrays: DEVICE. */
typedef struct {
  const int32_t *q_start; /* [n_seqs + 1] */
  const int32_t *kv_len;  /* [n_seqs] */
  const int32_t *pages;   /* [n_seqs][pages_stride] */
  int64_t pages_stride;
  int32_t max_pages;      /* entries of a row of pages, at least 1, at most pages_stride where there are more sequences than one;
                             max_pages * page_size at most 2^30 (PPD_ELIMIT) */
  int32_t n_seqs;         /* 1 .. PPD_MAX_SEQS */
  int32_t n_tokens;       /* rows of the batch's tensors, 0 .. PPD_MAX_TOKENS (0: nothing is done) */
} ppd_paged_batch;

/* Rows [n_tokens][heads][head_dim] with strides in elements; every row of head_dim elements begins at a multiple of 16 bytes. */
typedef struct {
  void *p;
  int64_t token, head;
} ppd_rows;

/* Queries and keys of the new tokens normalised per head and rotated to their positions, keys and values written to
 * their pages, in one pass.
 *   x' = x * rsqrt(mean(x^2) + norm_eps) * gain            where a gain is given (q_gain, k_gain: DEVICE, [head_dim], of
 *                                                          the cache's dtype, 8-byte aligned (fp32: 16); NULL: x' = x)
 *   (x'_i, x'_{i + r/2}) turned by position * rope_theta^(-2 i / r), i < r/2, r = rotary_dim (a multiple of 8 up to
 *                                                          head_dim; 0: nothing is turned)
 * Angles are reduced in 64 bits, everything else is fp32 with one rounding at the end; values are copied as they are.
 * q, q_out: n_heads heads (n_heads 0 and NULL, NULL: keys and values only).  q_out may be q itself (the same strides);
 * otherwise no output overlaps an input.  Queries are computed for every row of a sequence, also where its position has
 * no page or is negative (kv_len[s] below the sequence's number of rows).  Two rows of a batch that fall on one slot
 * (sequences that share a page they write to) race for it. */
int ppd_paged_append(const ppd_paged_cache *cache, const ppd_paged_batch *batch, int n_heads, const ppd_rows *q,
                     const ppd_rows *q_out, const ppd_rows *k, const ppd_rows *v, const void *q_gain,
                     const void *k_gain, float norm_eps, int rotary_dim, float rope_theta, void *hip_stream);

/* Attention of the new tokens over their sequences' pages: query head h reads key/value head h / (n_heads / n_kv_heads)
 * (n_heads a multiple of n_kv_heads; PPD_ELIMIT where n_tokens * n_heads / n_kv_heads passes 2^26, or a launch would have 2^24
 * workgroups: from about n_tokens * n_heads = 2^28 on, 2^31 for long runs of 16-bit types),
 *   out = sum_j softmax_j(scale * q . k_j) v_j
 * over the sequence's positions j up to the row's own (the new tokens' keys and values are in the pages already) and, with
 * window > 0, the last `window` of them only, its own included.  scale > 0, at most 2^127 (fp32: scale * log2 e times
 * each component of a query has to be finite, too).  A row that sees no position gives zeros.  What a row does not see
 * has no part in its result, whatever its bits (infinities, NaN, pages of other sequences).  out may be q itself (the
 * same strides), and overlaps no other input.
 * lse: DEVICE float [n_tokens][n_heads] or NULL: log of the sum of exp(scale * q . k_j), -inf where nothing is seen (for
 * a merge with attention over other positions).
 * Scores, softmax and sums are fp32; a 16-bit type's softmax weights go into their product with the values as two terms
 * of the type, so that the result's own rounding is what counts.  Beyond the order of additions (a sequence's positions
 * are cut into as many parts as the batch leaves compute units for) results do not depend on what else is in the batch,
 * and two calls with the same arguments give the same bits.
 * workspace: DEVICE scratch of at least the bytes that ppd_paged_attention_workspace gives for the same arguments (it
 * depends on sizes only, not on lengths), 16-byte aligned; NULL where those are 0.  PPD_EINVAL if workspace_bytes is less. */
int ppd_paged_attention(const ppd_paged_cache *cache, const ppd_paged_batch *batch, int n_heads, const ppd_rows *q,
                        const ppd_rows *out, float *lse, float scale, int window, void *workspace,
                        uint64_t workspace_bytes, void *hip_stream);
int ppd_paged_attention_workspace(const ppd_paged_cache *cache, const ppd_paged_batch *batch, int n_heads,
                                  uint64_t *bytes);

/* Drafted tokens against the target model, by the rule of speculative sampling: every emitted token is distributed as the
 * target's own.  Rows are those of the batch that went through the target: sequence s has rows row_start[s] ..
 * row_start[s+1]-1 (none: it takes no part), ids[row] is the token that went in: the sequence's last token, then its
 * drafts.  target_logits [n_rows][vocab] (rows target_stride elements apart): row r's prediction of the token behind it.
 * draft_logits, likewise: row r holds the distribution that ids[r + 1] was drawn from (a sequence's last row is not
 * read), or NULL: the drafts were not drawn (an arg max, an early prediction's candidate).
 *   p = softmax(target_logits[r] / t), q = softmax(draft_logits[r] / t) (NULL: q = 1 at ids[r + 1]), t = temperature[s]
 *   the draft d = ids[r + 1] is taken if uniform[r][0] * q(d) < p(d);
 *   at the first row whose draft is not taken the token is drawn from max(p - q, 0) (from p where that is 0 everywhere),
 *   and behind the last draft, all being taken, from p: the lowest id whose cumulative mass, in id order, exceeds
 *   uniform[r][1] times the whole.
 * temperature: DEVICE float [n_seqs], or NULL: 1 for all.  t <= 0 (or NaN): arg max, ties to the lowest id; a draft is
 * taken if it is the arg max, and neither draft_logits nor uniform have a say.  Probabilities and their sums are fp64;
 * those below 2^-900 of the largest count as 0.  Logits of -inf and NaN have probability 0 (tokens that top-k or top-p
 * filtering took out); a row of nothing else takes no draft and gives token 0, as an arg max of it does; +inf counts as
 * the type's largest finite number would in fp32 (tokens that have it share the row).  Drafts outside [0, vocab) are not
 * taken.  uniform: DEVICE float [n_rows][2] in [0, 1).
 * Out, DEVICE: tokens int32 [n_rows]: at a sequence's rows the drafts taken, then the drawn token, then -1; accepted
 * int32 [n_seqs]: the number of drafts taken (the sequence gained that many tokens and one more; 0 for one without
 * rows).  Rows of no sequence are not touched; no output overlaps an input.  vocab 1 .. 2^24, n_rows 0 ..
 * PPD_MAX_TOKENS, n_seqs 1 .. PPD_MAX_SEQS, n_rows * ceil(vocab / 4096) at most 2^23.
 * target_logits and draft_logits of type dtype, aligned to it (any stride of at least vocab).  workspace as above, from
 * ppd_verify_drafts_workspace. */
int ppd_verify_drafts(int n_seqs, int n_rows, int vocab, int dtype, const int32_t *row_start, const int32_t *ids,
                      const void *target_logits, int64_t target_stride, const void *draft_logits, int64_t draft_stride,
                      const float *temperature, const float *uniform, int32_t *tokens, int32_t *accepted,
                      void *workspace, uint64_t workspace_bytes, void *hip_stream);
int ppd_verify_drafts_workspace(int n_seqs, int n_rows, int vocab, int dtype, uint64_t *bytes);

#ifdef __cplusplus
}
#endif
#endif /* PPD_LAYERS_H */
