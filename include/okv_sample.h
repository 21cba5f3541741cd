/*
 * okv_sample -- from logits to tokens, for one MI355X: probabilities, and drafted tokens held against them.
 *
 * Conventions as in okv.h: C ABI, every pointer DEVICE unless labelled, the caller owns all memory, calls enqueue on `stream` and
 * return at once without allocating, copying or waiting (all may be captured in a graph); OKV_OK or a negative OKV_E* code;
 * okv_last_error(NULL) has the message.
 */
#ifndef OKV_SAMPLE_H
#define OKV_SAMPLE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define OKV_SAMPLE_MAX_VOCAB (1 << 24)
#define OKV_SAMPLE_MAX_ROWS (1 << 20)
#define OKV_VERIFY_MAX_BATCH 4096

/* out[r][i] = softmax_i(logits[r][i] / t_r), sums in fp32.
 *   logits       fp16 (dtype 0) or fp32 (1) [rows][vocab], rows `stride` elements apart (at least vocab), aligned to their size
 *   temperature  fp32 [rows], or NULL: 1.  0: 1 at the first of the row's largest logits, 0 elsewhere.  Infinite: the same for every logit above
 *                -infinity.  Negative or NaN: the row is NaN
 *   out          fp32 [rows][vocab], rows out_stride elements apart; not overlapping logits
 * A logit of -infinity has probability 0, a row of nothing else is 0.  One that is infinite or NaN makes its row NaN (an infinite
 * one at temperature 0 is the largest, and NaN is passed over there). */
int okv_token_probs(const void *logits, int32_t dtype, int64_t stride, const float *temperature, float *out, int64_t out_stride, int32_t rows, int32_t vocab,
                    void *workspace, int64_t workspace_bytes, void *stream);

/* Workspace of okv_token_probs for up to this many rows (16-byte aligned); < 0 on a bad shape. */
int64_t okv_token_probs_workspace_bytes(int32_t max_rows, int32_t vocab);

/* Drafted tokens against the target's probabilities.  Sequence b has n = starts[b + 1] - starts[b] drafts x_0 .. x_{n-1}, drawn from q_0 .. q_{n-1}, and
 * n + 1 rows p_0 .. p_n of the target, the first at row starts[b] + b; as many random numbers u_0 .. u_n lie there.
 *   x_i is accepted as long as u_i q_i(x_i) < p_i(x_i), the product in fp32; the first that is not, x_a, and those behind it are
 *   rejected (none: a = n).  A token outside [0, vocab) is rejected.
 *   The next token is drawn with u_n: with weights w = max(p_a - q_a, 0) if a < n (p_a where they are all 0), w = p_n if a = n, it is the first t
 *   with w_0 + .. + w_t > u_n (w_0 + .. + w_{vocab-1}).  Differences and sums are in 64 bits; weights that are not positive or not finite count as 0.
 *   If all weights are 0 the token is -1.
 *   With draft_probs NULL the drafts are certain: q_i is 1 at x_i and 0 elsewhere.
 *
 *   target       fp32 [n_rows + batch][vocab], rows target_stride elements apart
 *   draft_probs  fp32 [n_rows][vocab], rows draft_stride apart, or NULL
 *   drafts       int32 [n_rows];  starts int32 [batch + 1], ascending from 0;  n_rows starts[batch], or more
 *   uniforms     fp32 [n_rows + batch], in [0, 1)
 *   tokens       int32 [n_rows + batch]: x_0 .. x_{a-1}, the next token, and -1 behind it, from starts[b] + b on
 *   accepted     int32 [batch]: a;  rejected  int32 [batch]: n - a, or NULL.  (With okv_pages_shrink the cache gives the rejected ones' pages back.)
 *   workspace    okv_verify_workspace_bytes(batch, vocab) bytes, 16-byte aligned; calls that may run at the same time need workspaces of their own */
int okv_verify(const float *target, int64_t target_stride, const float *draft_probs, int64_t draft_stride, const int32_t *drafts, const int32_t *starts,
               const float *uniforms, int32_t *tokens, int32_t *accepted, int32_t *rejected, int32_t batch, int32_t n_rows, int32_t vocab,
               void *workspace, int64_t workspace_bytes, void *stream);
int64_t okv_verify_workspace_bytes(int32_t max_batch, int32_t vocab);

#ifdef __cplusplus
}
#endif
#endif /* OKV_SAMPLE_H */
