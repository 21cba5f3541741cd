/*
 * okv_chunk -- several new tokens of a sequence at once over the fp16 cache of okv.h, for one MI355X.
 *
 * A prompt that is stored in chunks, tokens that a draft has proposed, or a batch in which some sequences bring a prompt
 * and others a token: the rows of every sequence go into the cache, their keys and queries turned by their
 * positions on the way (okv_rope_append), and every row attends over its sequence up to itself (okv_chunk_attn).
 * okv_decode_attn_static is the step of one token per sequence; it reads the same pools.
 *
 * Conventions as in okv.h: C ABI, every pointer DEVICE unless labelled, the caller owns all memory, calls enqueue on the
 * stream and return at once; OKV_OK or a negative OKV_E* code; okv_last_error(NULL) has the message.  No call
 * allocates, copies or waits: all may be captured in a graph.  Lengths, starts, rows of the table and page numbers are read
 * on the device: a length is taken as at least 0, what lies past the capacity is not there, wrong rows of the table are passed
 * over, nothing is stored in wrong pages and reading them gives wrong numbers, no access outside the buffers.
 */
#ifndef OKV_CHUNK_H
#define OKV_CHUNK_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define OKV_CHUNK_MAX_BATCH 4096

/* One layer of an fp16 cache, laid out as okv.h says. */
typedef struct okv_layer_pool {
  int32_t n_q_heads, n_kv_heads, head_dim;   /* H, G, d as in okv_config: H % G == 0, H / G <= 16, d 64 or 128          */
  int32_t block_tokens;                      /* T: 0 = contiguous, else a power of two in [16, 1024]                    */
  int32_t max_blocks_per_seq;                /* paged: columns of block_table                                           */
  int32_t max_ctx;                           /* contiguous: capacity in tokens per sequence, a multiple of 16           */
  int32_t max_seqs;                          /* rows of block_table, or sequences of a contiguous pool                  */
  int64_t n_blocks;                          /* paged: blocks of the pool                                               */
  void *pool;                                /* the layer's K and V, 16-byte aligned                                    */
  const int32_t *block_table;                /* [max_seqs][max_blocks_per_seq]; contiguous: ignored                     */
  const int32_t *refused;                    /* NULL, or a word: while it is not 0 nothing is written to the pool
                                                (status + 3 of okv_pages.h: pages could not be taken, and the
                                                caller has not seen it yet)                                            */
} okv_layer_pool;

/* Which rows are whose: those of a call over `batch` sequences, one sequence's after the other's.
 *   seqs    [batch] rows of block_table (distinct), or NULL: sequence b is row b
 *   starts  [batch + 1] ascending from 0: rows starts[b] .. starts[b + 1] - 1 are sequence b's, the last of its tokens
 *   lens    [max_seqs], by row of block_table: tokens that the sequence has, these rows included
 *   n_rows  starts[batch], or more (rows from starts[batch] on are neither read nor written) */
typedef struct okv_rows {
  int32_t batch;               /* 0 .. OKV_CHUNK_MAX_BATCH; 0: nothing is done */
  int32_t n_rows;
  const int32_t *seqs, *starts, *lens;
} okv_rows;

/* The turn of a row at position p: pair j of the first `rotated` elements of a head, (x, y), becomes
 *     (x cos a - y sin a, x sin a + y cos a),   a = 2 pi p turns[j]
 * with p turns[j] taken in 64 bits less its whole turns: positions of millions lose nothing.  Elements from `rotated` on stay. */
typedef struct okv_rope {
  const double *turns;         /* [rotated / 2]: turns per position                                                     */
  int32_t rotated;             /* a multiple of 16, at most d                                                           */
  int32_t interleaved;         /* pair j is elements 2 j and 2 j + 1; 0: elements j and j + rotated / 2                 */
  const int32_t *positions;    /* [n_rows] positions, or NULL: the row's token's place in its sequence                  */
} okv_rope;

/* Row i of n rows of a sequence of len tokens becomes its token len - n + i: keys turned, values as they are.  Tokens before 0
 * or past the capacity (a len may be above it) are not stored; their queries are turned by their positions all the same.
 *   k, v   fp16 [n_rows][G][d], rows kv_stride elements apart (a multiple of 8, at least G * d), 16-byte aligned
 *   q      fp16 [n_rows][H][d] (q_stride likewise) and q_out (q_out_stride): turned queries; NULL: there are none.  q_out may be q
 *          (with the same stride), and overlap nothing else
 *   rope   NULL: keys are stored, and queries copied, as they are */
int okv_rope_append(const okv_layer_pool *c, const okv_rows *r, const okv_rope *rope, const void *k, const void *v, int64_t kv_stride,
                    const void *q, int64_t q_stride, void *q_out, int64_t q_out_stride, void *stream);

/* Attention of every row over its sequence.  A row of the token at position p sees the keys i <= p, with a window only those above p - window, and
 * those below the sequence's prefix, wherever they are.  Scores, in fp32:
 *     s_i = scale (q . k_i);   s_i = cap tanh(s_i / cap) with a cap;   s_i -= slopes[h] |p - i| with slopes
 *     out = sum_i softmax_i(s) v_i
 * A row that sees no key is 0 (p < 0: the sequence has fewer tokens than rows).  Rows of tokens past the capacity (a len may be above it) attend as
 * the last token within it does.  A score of -infinity leaves its key out (0 if no key is left), one that is +infinity or NaN makes the row NaN; an infinite or NaN value makes the rows that see its key infinite or NaN in that
 * element, whatever the key's weight, 0 included.  What lies at keys that a row does not see, infinities and NaN included, does not
 * change it.  Weights are fp16 in the second product for an fp16 result (each off by 2^-11 of itself at most, or 2^-32 of the largest), two fp16
 * numbers for an fp32 one (2^-22); sums are fp32. */
typedef struct okv_chunk {
  float scale;                 /* 0: 1 / sqrt(d); else in [1e-30, 1e30]                                                 */
  float cap;                   /* 0: none; else in [1e-30, 1e30]                                                        */
  int32_t window;              /* 0: none                                                                               */
  const float *slopes;         /* [H], or NULL                                                                          */
  const int32_t *prefix;       /* [max_seqs], by row of block_table, or NULL                                            */
  int32_t out_dtype;           /* 0 = fp16, 1 = fp32                                                                    */
  void *workspace;             /* okv_chunk_workspace_bytes bytes, 256-byte aligned; calls that may run at the same time
                                  need workspaces of their own; its contents mean nothing between calls                 */
  int64_t workspace_bytes;
} okv_chunk;

/* q fp16 [n_rows][H][d], rows q_stride elements apart (a multiple of 8, at least H * d); out [n_rows][H][d] contiguous, not overlapping q. */
int okv_chunk_attn(const okv_layer_pool *c, const okv_rows *r, const okv_chunk *a, const void *q, int64_t q_stride, void *out, void *stream);

/* Workspace for any batch on this shape of pool (pool and tables are not looked at); < 0 on a bad shape. */
int64_t okv_chunk_workspace_bytes(const okv_layer_pool *c);

#ifdef __cplusplus
}
#endif
#endif /* OKV_CHUNK_H */
