/*
 * okv8 -- a paged KV cache held in 8 bits, and decode attention over it, for one MI355X.
 *
 * Decode attention reads the whole cache once per step and is bound by doing so (paper §IV-D: one flop
 * per cached byte), and what of the cache does not fit in GPU memory crosses the host link every step
 * (§II-B).  Half the bytes are half of both.  The fp16 cache of okv.h and this one are separate: a
 * program uses either.
 *
 * What is held.  32 consecutive tokens of a sequence (tokens 32 t .. 32 t + 31) are a TILE.  For every
 * tile, KV head, and K or V by itself, with a = max |x| over the 32 * d numbers:
 *     scale = a * (1 / M)      M = 127 (OKV8_INT8) or 448 (OKV8_E4M3); 1 / M and the product in fp32,
 *                              the result rounded up to 12 significant bits
 *     code  = x / scale        to nearest, ties to even; a whole number, or an OCP E4M3 value
 *     (a = 0: scale 0, codes 0;  a number that is infinite or NaN: scale NaN, so that everything that
 *     reads the tile is NaN)
 * Rounding the scale up keeps |code| <= M, and with 12 bits the fp32 quotient is on the right side of
 * every rounding boundary (a boundary times the scale has at most 21 bits, x has 11, so a quotient that
 * is not on the boundary is 2^-21 away from it): codes are the exact ones, whoever computes them.
 * The tokens of a sequence's last tile, as long as it is not full, stay in fp16 in 32 rows per sequence,
 * its TAIL: a tile is quantised once, when it is full, from the numbers as they came.  Storing a prompt
 * and appending it token by token leave the same bits.
 *
 * Layout (G KV heads, d = head_dim, T = page_tokens; layers one after the other in each buffer)
 *   codes   [L][n_pages][T / 32][G / Gg][kv][Gg][32 * d] bytes     kv = 0 keys, 1 values
 *           Gg = okv_kv_head_group(G, d).  The 32 * d bytes of a tile and head are in the order in which
 *           lanes of a wavefront feed them to the matrix cores, 16 bytes a lane:
 *             K: byte 16 (64 j + lane) + 8 p + i, j = 2 h + c / 2 at d = 128 (j = h at 64), p = c % 2:
 *                key 16 h + lane % 16, element 32 c + 8 (lane / 16) + i
 *             V: byte 16 (64 j + lane) + 8 p + i: element 16 (2 j + p) + lane % 16 of
 *                key 4 (lane / 16) + i (i < 4) or 16 + 4 (lane / 16) + i - 4
 *           OKV8_INT8 codes are stored as code + 128, OKV8_E4M3 codes as they are.
 *   scales  [L][n_pages][T / 32][G][kv] fp32
 *   tails   [L][max_seqs][kv][G][32][d] fp16, token i in row i % 32
 *   page_table [max_seqs][max_pages_per_seq] int32: token i of sequence s is in page
 *           page_table[s][i / T].  Pages may be shared by sequences as long as only full tiles are in
 *           them (okv_pages.h forks sequences that way).
 *
 * Conventions as in okv.h: C ABI, every pointer DEVICE unless labelled, 16-byte aligned, the caller owns
 * all memory, calls enqueue on the stream and return at once; OKV_OK or a negative OKV_E* code;
 * okv_last_error(NULL) has the message.  No call allocates, copies or waits: all may be captured in a
 * graph.  Lengths and page numbers are read on the device; a length is taken as at least 0 and at most
 * max_pages_per_seq * T and a page as in [0, n_pages): wrong ones give wrong numbers, no access outside
 * the buffers.  The same holds for entries of `seqs`, which must be in [0, max_seqs) and distinct.
 */
#ifndef OKV_CACHE8_H
#define OKV_CACHE8_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define OKV8_INT8 0
#define OKV8_E4M3 1
#define OKV8_TILE 32
#define OKV8_MAX_BATCH 4096

typedef struct okv8_cache {
  int32_t n_layers;            /* L >= 1                                                     */
  int32_t n_q_heads;           /* H; H % G == 0 and 1 <= H / G <= 16                         */
  int32_t n_kv_heads;          /* G in [1, 1024]                                             */
  int32_t head_dim;            /* d in {64, 128}                                             */
  int32_t page_tokens;         /* T: a power of two in [32, 1024]                            */
  int32_t format;              /* OKV8_INT8 or OKV8_E4M3                                     */
  int32_t out_dtype;           /* of the attention output: 0 = fp16, 1 = fp32                */
  int32_t max_seqs;            /* rows of page_table and of tails                            */
  int32_t max_pages_per_seq;   /* columns of page_table                                      */
  int64_t n_pages;             /* pages of every layer, at most 2^31 - 1                     */
  void *codes, *scales, *tails;
  const int32_t *page_table;
  const int32_t *refused;      /* NULL, or a word: while it is not 0, storing writes nothing, and a step that
                                  appends writes nothing to the cache (its results then mean nothing).
                                  status + 3 of okv_pages.h: pages could not be taken, and the caller has
                                  not seen it yet                                            */
} okv8_cache;

/* Bytes of the three buffers (all layers); < 0 on a bad shape. */
int64_t okv8_codes_bytes(const okv8_cache *c);
int64_t okv8_scales_bytes(const okv8_cache *c);
int64_t okv8_tails_bytes(const okv8_cache *c);

/* Stores rows of `batch` sequences in layers layer .. layer + n_layers - 1, in one launch.
 *   seqs    [batch] rows of page_table, or NULL: sequence b is row b
 *   starts  [batch + 1] ascending from 0: rows starts[b] .. starts[b + 1] - 1 are sequence b's
 *   lens    [max_seqs], by row of page_table: tokens that the sequence has AFTER the call; its rows are
 *           the last ones of them.  Tokens before them are there already (a tile that the call fills takes
 *           its first rows from the tail).
 *   n_rows  starts[batch]; rows beyond it are not read.  0: nothing is done
 *   k, v    fp16 [n_layers][n_rows][G][d]; row_stride elements from a row to the next (a multiple of 8, at
 *           least G * d), layer_stride from a layer to the next (a multiple of 8) */
int okv8_store(const okv8_cache *c, int32_t layer, int32_t n_layers, int32_t batch, const int32_t *seqs,
               const int32_t *starts, const int32_t *lens, int64_t n_rows, const void *k, const void *v,
               int64_t row_stride, int64_t layer_stride, void *stream);

/* The reverse: the last starts[b + 1] - starts[b] of lens[] tokens of every sequence as the cache holds
 * them (code * scale rounded to fp16, or the tail's rows), into k and v, shaped as for okv8_store.  (A tile's largest number may be held up to
 * 2^-11 of it too large: fp16's largest, 65504, comes out as an infinity.) */
int okv8_load(const okv8_cache *c, int32_t layer, int32_t n_layers, int32_t batch, const int32_t *seqs,
              const int32_t *starts, const int32_t *lens, int64_t n_rows, void *k, void *v,
              int64_t row_stride, int64_t layer_stride, void *stream);

/* One decode step of a batch. */
typedef struct okv8_step {
  int32_t batch;               /* 1 .. min(max_seqs, OKV8_MAX_BATCH)                         */
  int32_t appends;             /* 1: every layer's call brings a row per sequence, which becomes
                                  token lens - 1;  0: the calls attend over what is there     */
  const int32_t *seqs;         /* [batch] or NULL, as above                                  */
  const int32_t *lens;         /* [max_seqs] keys that are attended, an appended one included.
                                  0: nothing is appended, the output is 0                    */
  void *workspace;             /* up to okv8_workspace_bytes(c, batch) bytes, 256-byte aligned */
  int64_t workspace_bytes;
  void *stream;
} okv8_step;

/* Workspace of a step of up to max_batch sequences; < 0 on a bad shape.  okv8_decode_step attends up to 32 layers in one launch
 * with it; what this returns for a cache of one layer is enough for okv8_decode_attn, and okv8_decode_step then takes fewer
 * layers at a time.  Its contents mean nothing between steps; from okv8_step_begin to the step's last okv8_decode_attn nothing else may use it
 * (okv8_decode_step included), and seqs and lens must stay as they are.  Steps that may run at the same time need
 * workspaces of their own. */
int64_t okv8_workspace_bytes(const okv8_cache *c, int32_t max_batch);

/* Shares the step's keys out over the wavefronts: once per step, before the first okv8_decode_attn. */
int okv8_step_begin(const okv8_cache *c, const okv8_step *s);

/* One layer: stores the appended rows and attends,
 *     out[b][h] = sum_i softmax_i(q[b][h] . k_i / sqrt(d)) v_i,   i < lens,  KV head h / (H / G)
 * An appending step reads the tokens before 32 floor((lens - 1) / 32) as their codes say and the others, the
 * appended one included, in fp16 from the tail, and then quantises a tail that is full; a step that appends
 * nothing reads the tokens before 32 floor(lens / 32) as their codes say.  Infinite numbers in the tail are taken for what they
 * are: a score of -infinity leaves its key out (NaN if no key is left), an infinite value makes the result infinite (NaN if its weight is
 * below 2^-31 of the largest, if the same element has the other infinity, or a NaN).
 *   q     fp16 [batch][H][d], q_stride elements from a sequence to the next (a multiple of 8)
 *   k_new, v_new  fp16 [batch][G][d], kv_stride likewise; both NULL if the step does not append
 *   out   [batch][H][d] in out_dtype */
int okv8_decode_attn(const okv8_cache *c, const okv8_step *s, int32_t layer, const void *q, int64_t q_stride,
                     const void *k_new, const void *v_new, int64_t kv_stride, void *out);

/* A step whose inputs are there for all layers, in one launch where a row of the page table holds at most 1024 keys and there are few of (layer, sequence,
 * KV head), otherwise in two, three beyond 64 sequences (okv8_step_begin and okv8_decode_attn for every layer
 * give the same up to the order in which partial results are added):
 * q [L][batch][H][d], k_new / v_new [L][batch][G][d] (or NULL), out [L][batch][H][d], all contiguous. */
int okv8_decode_step(const okv8_cache *c, const okv8_step *s, const void *q, const void *k_new,
                     const void *v_new, void *out);

#ifdef __cplusplus
}
#endif
#endif /* OKV_CACHE8_H */
