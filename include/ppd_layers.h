/* Operators of libppd for programs that run a model's layers themselves, beside ppd_early_topk (ppd.h): the keys and
 * values of many sequences in pages, the attention of new tokens over them, and the verification of drafted tokens
 * against the target model's logits.  Together they make a step that checks drafts: the last token and the drafts of
 * every sequence go through the layers as one ragged batch (ppd_paged_append and ppd_paged_attention in each), and
 * ppd_verify_drafts turns the logits of all their rows into the tokens to emit.  What a rejected draft left in the
 * pages needs no undoing: the next step's tokens are written over it.
 * ppd_paged_plan makes a step's batch (rows, lengths, pages) on the device from what the step before has left,
 * ppd_adjust_logits comes between the logits and their verification, and ppd_paged_append_fp4 and
 * ppd_paged_attention_fp4 are the two operators on pages for keys and values of 4 bits.
 *
 * All only queue their work on hip_stream (a hipStream_t of the current device, NULL = its default stream): they
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

/* A step's batch, made on the device: how many tokens each sequence adds, the pages that it gives back or takes, and
 * where its rows lie.  A sequence of the table has `held` positions (their pages are the table's first ceil(held /
 * page_size) places), keeps the first `kept` of them (drafts that were not taken go; 0: all, the sequence has ended) and
 * asks for `wanted` more.  It gets all of them or none:
 *   none where kept + wanted is more than max_pages * page_size;
 *   none where it and the sequences before it (but for those of the line above) ask for more than n_rows tokens;
 *   none where it needs pages, and it and the sequences before it (but for those of the lines above) need more than
 *   there are free ones.
 * The table is changed in place: places that kv_len = kept + granted needs no more are given back (their entries stay),
 * places that it needs and held did not are filled.  Free pages are a ring of n_pages numbers, free_pages: counters[0]
 * pages were taken since it was made and counters[1] put in; number i lies at place i modulo n_pages, so counters[1] -
 * counters[0] are free.  (A pool of which all pages are free: 0 .. n_pages-1, counters 0 and n_pages.)  Pages are taken, and put
 * in, in the order of sequences and of their places; what a call puts in can be taken from the next call on.
 * A page belongs to one sequence.  Entries outside [0, n_pages) are given back by no one; counters that lie as no call
 * leaves them count as a ring that holds nothing (fewer than 0 free) or n_pages (more).
 * Lengths outside their range count as the next number inside: held within the table's room, kept within [0, held],
 * wanted at least 0.
 * Out, DEVICE: q_start [n_seqs + 1], kv_len [n_seqs] and granted [n_seqs] (tokens of each sequence); counters_out [2]; and,
 * each of them unless NULL, for every row of [0, n_rows) row_seq, positions (in the sequence) and slots (page *
 * page_size + place in it), all -1 for rows of no sequence, slots -1 too where the entry is no page.
 * kv_len may be held itself and counters_out counters; no other two tensors overlap.  held, kept (NULL: all stay), wanted:
 * DEVICE int32 [n_seqs]. */
typedef struct {
  int32_t *pages;         /* [n_seqs][pages_stride] */
  int64_t pages_stride;   /* at least max_pages where there are more sequences than one */
  int32_t *free_pages;    /* [n_pages] */
  int32_t max_pages;      /* at least 1; max_pages * page_size and n_seqs * max_pages at most 2^30 (PPD_ELIMIT) */
  int32_t n_pages;        /* at least 1 */
  int32_t page_size;      /* at least 1 */
  int32_t n_seqs;         /* 1 .. PPD_MAX_SEQS */
} ppd_page_table;

int ppd_paged_plan(const ppd_page_table *table, const int64_t *counters, int64_t *counters_out, const int32_t *held,
                   const int32_t *kept, const int32_t *wanted, int n_rows, int32_t *q_start, int32_t *kv_len,
                   int32_t *granted, int32_t *row_seq, int32_t *positions, int64_t *slots, void *hip_stream);

/* Keys and values of 4 bits in pages (the MX format: elements e2m1, scales e8m0).  A row of head_dim numbers is head_dim / 2 bytes
 * of codes, element 2i in the low half of byte i, and head_dim / 32 scales, one byte for 32 elements in a row: bit 3 of a
 * code is its sign, the others stand for 0, 0.5, 1, 1.5, 2, 3, 4, 6, and scale b multiplies by 2^(b - 127) (from 253 on: the 32
 * numbers are NaN).  k, v: [n_pages][page_size][n_kv_heads][head_dim / 2],
 * k_scales, v_scales: [n_pages][page_size][n_kv_heads][head_dim / 32], each in any order of the first three that its
 * strides (in BYTES) express, the last contiguous (a head's positions side by side are read fastest); strides of 0: for
 * ppd_paged_attention_fp4 only.  Rows of codes begin at
 * multiples of 16 bytes, rows of scales at multiples of head_dim / 32 (so do the tensors, and so do all strides). */
typedef struct {
  void *k, *v, *k_scales, *v_scales;
  int64_t k_page, k_pos, k_head, v_page, v_pos, v_head;
  int64_t ks_page, ks_pos, ks_head, vs_page, vs_pos, vs_head;
  int32_t n_pages;
  int32_t page_size;  /* positions of a page, at least 1 */
  int32_t n_kv_heads;
  int32_t head_dim;   /* 64 or 128 */
  int32_t dtype;      /* PPD_FP32, PPD_BF16, PPD_FP16: of the rows of queries, keys, values and outputs that go in and come out */
} ppd_paged_cache_fp4;

/* ppd_paged_append into such pages: queries and keys normalised and rotated as there, keys and values to the nearest numbers
 * that the pages can hold.  32 numbers x get the least scale 2^e, e in [-125, 125], with max|x| <= 7 * 2^e (7 rounds to 6, no
 * further off than half a step), and each the nearest code, ties to the even one; what is beyond 7 * 2^125 becomes 6 * 2^125.
 * 32 numbers with an infinity or NaN among them: scale 255, codes 0.  Keys are worked out in 64 bits up to their
 * codes, so that which code it is does not depend on an order of operations; queries as in ppd_paged_append.
 * k_out, v_out: rows like k and v (or NULL): the keys and values as the pages have them now, rounded to the type (for
 * attention over the batch's own rows, say); like q_out they are written for every row of a sequence, with a page or without.
 * q_out may be q itself, k_out k and v_out v (the same strides); otherwise no output overlaps an input or another output.
 * Everything else as in ppd_paged_append. */
int ppd_paged_append_fp4(const ppd_paged_cache_fp4 *cache, const ppd_paged_batch *batch, int n_heads, const ppd_rows *q,
                         const ppd_rows *q_out, const ppd_rows *k, const ppd_rows *v, const ppd_rows *k_out,
                         const ppd_rows *v_out, const void *q_gain, const void *k_gain, float norm_eps, int rotary_dim,
                         float rope_theta, void *hip_stream);

/* ppd_paged_attention over such pages: the same arguments, rules and limits.  Keys and values are taken as bf16 numbers,
 * which they are without rounding; queries of fp16 and fp32, and softmax weights, go into their products as two or three bf16 terms, so
 * that as there the result's own rounding is what counts (fp32: of 24 bits).  Queries are finite numbers. */
int ppd_paged_attention_fp4(const ppd_paged_cache_fp4 *cache, const ppd_paged_batch *batch, int n_heads, const ppd_rows *q,
                            const ppd_rows *out, float *lse, float scale, int window, void *workspace,
                            uint64_t workspace_bytes, void *hip_stream);
int ppd_paged_attention_fp4_workspace(const ppd_paged_cache_fp4 *cache, const ppd_paged_batch *batch, int n_heads,
                                      uint64_t *bytes);

/* Logits as a request wants them, before ppd_verify_drafts or a sampler of one's own.  Rows, row_start and ids as there: row
 * r of sequence s predicts the token behind ids[r].  Its text is history[s][0 .. history_len[s]-1], the tokens before
 * the batch's, and then ids[row_start[s]] .. ids[r].  In this order, in fp32 and with one rounding at the end, for token t of row r:
 *   x = logits[r][t]
 *   repetition: if t is in the text, x = x > 0 ? x * (1 / repetition[s]) : x * repetition[s]   (a number that is not above 0: x as it is)
 *   frequency, presence: if t is n > 0 times in the text behind its first prompt_len[s] tokens, x -= frequency[s] * n + presence[s]
 *   bias: x += bias[e] for the last e in [bias_start[s], bias_start[s+1]) with bias_ids[e] = t
 *   mask: if bit t % 32 of word mask[mask_row[r]][t / 32] is 0, x = -inf   (mask_row[r] outside [0, n_masks): all tokens are allowed)
 * Tokens outside [0, vocab) in the text or the biases are none.  history_len counts as within [0, history_stride], bias_start
 * as within [0, n_bias].  out: like logits, may be logits itself (the same stride); no other tensor overlaps out.  Rows of no
 * sequence are not touched (row_start must not decrease, as q_start there).
 * All of it DEVICE, contiguous but for the rows' strides (in elements), and each of these may be NULL: ids (the text is the history), history
 * and history_len (both: the text is the batch's rows), prompt_len (0), repetition (1), presence (0),
 * frequency (0), bias_start, bias_ids and bias (all three), mask and mask_row (both).  With n_rows 0 nothing is done, and logits, out and
 * mask_row may be NULL, too. */
typedef struct {
  const int32_t *history;       /* [n_seqs][history_stride] */
  int64_t history_stride;       /* at most 2^30 */
  const int32_t *history_len, *prompt_len;                 /* [n_seqs] */
  const float *repetition, *presence, *frequency;          /* [n_seqs] */
  const int32_t *bias_start;    /* [n_seqs + 1] */
  const int32_t *bias_ids;      /* [n_bias] */
  const float *bias;            /* [n_bias] */
  const uint32_t *mask;         /* [n_masks][mask_stride] */
  int64_t mask_stride;          /* words, at least ceil(vocab / 32) */
  const int32_t *mask_row;      /* [n_rows] */
  int32_t n_bias, n_masks;
} ppd_logit_rules;

/* vocab 1 .. 2^24, n_rows 0 .. PPD_MAX_TOKENS, n_seqs 1 .. PPD_MAX_SEQS, strides of at least vocab, logits and out of type dtype and aligned
 * to it. */
int ppd_adjust_logits(int n_seqs, int n_rows, int vocab, int dtype, const int32_t *row_start, const int32_t *ids,
                      const void *logits, int64_t logits_stride, void *out, int64_t out_stride,
                      const ppd_logit_rules *rules, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PPD_LAYERS_H */
