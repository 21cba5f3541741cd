/*
 * okv_pages -- pages of a paged KV cache: taking, forking, shortening, freeing, compacting and copying them, on one
 * MI355X.
 *
 * A cache whose pages are runs of bytes, the same number for every page, can be managed here: the fp16
 * pools of okv.h in blocks (block_tokens > 0, attended with okv_decode_attn_static, whose tables are
 * DEVICE arrays too) and the 8-bit cache of okv_cache8.h.  All state is on the GPU, so that a step that
 * takes, forks or frees pages needs no copy from the host and can be captured in a graph.
 *
 *   table  [max_seqs][max_pages_per_seq] int32: page of token i of sequence s = table[s][i / T], -1: none
 *   lens   [max_seqs] int32: tokens of every sequence; its first ceil(lens / T) entries are its pages
 *   refs   [n_pages] int32: sequences that a page belongs to; 0: free.  Start with table -1, lens and refs 0.
 *   status [4] int32: 0 or the code of the first call that could not be carried out (the caller clears
 *          it); [1] pages in use after the last okv_pages_compact; [2] pages that it moved; [3] 0 or the
 *          code of the last okv_pages_extend (the caller may clear it), which stays as long as status[0]
 *          is not cleared
 *
 * A page that several sequences share is full and is never written: a fork copies the last, partly
 * filled page.  Free pages are taken lowest id first, in the order of the arguments.  Whether there are
 * enough is known on the GPU only: a call that lacks pages, or room in a row of the table, changes
 * nothing and leaves OKV_ENOSPC in status[0], one whose arguments do not fit the state OKV_ESTATE; a
 * program that cannot rule this out reads status[0] when it next synchronises.  After an okv_pages_extend that was
 * refused, later ones change nothing either, whatever their sequences, until the caller has cleared
 * status[0]: no sequence has tokens that no step has written.  A step that follows an
 * okv_pages_extend which changed nothing must not append: the row would go where the last token is, which
 * may be in a shared page.  A step over the 8-bit cache sees to that itself (okv8_cache.refused), and so does storing rows; a program
 * that appends to an fp16 pool reads status[3] first, unless it knows that there are pages.
 *
 * Conventions as in okv.h: C ABI, every pointer DEVICE unless labelled, the caller owns all memory,
 * calls enqueue on `stream` and return at once without allocating; OKV_OK or a negative OKV_E* code;
 * okv_last_error(NULL) has the message.  Row numbers and page ids are checked on the GPU: wrong ones are
 * passed over.  Calls on one cache must follow one another on one stream.
 */
#ifndef OKV_PAGES_H
#define OKV_PAGES_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define OKV_PAGES_MAX_ARRAYS 4
#define OKV_PAGES_MAX_ROWS   2
#define OKV_PAGES_MAX_SEQS   4096      /* sequences per call                                          */

/* What a page holds: page p of layer l is page_bytes bytes at base + l * layer_stride + p * page_bytes.
 * It is a row of T / unit_tokens units; a fork copies the units of the last page that hold tokens: those
 * that are partly filled as well, or, with whole_units, only full ones (what a partly filled unit holds is
 * kept per sequence, in an okv_row_array).  page_bytes, layer_stride, base and the bytes of a unit must be multiples of 4;
 * where they all are of 16, 16 bytes are moved at a time. */
typedef struct okv_page_array {
  void *base;
  int64_t page_bytes, layer_stride;
  int32_t unit_tokens, whole_units;
} okv_page_array;

/* What a sequence holds beside its pages: `groups` groups of `rows` rows of row_bytes bytes, sequence s of layer l at
 * base + l * layer_stride + s * groups * rows * row_bytes; token i is in row i % rows of every group.  A fork copies the
 * first lens % rows rows of each.  Multiples of 4 and 16 as above. */
typedef struct okv_row_array {
  void *base;
  int64_t layer_stride;
  int32_t groups, rows, row_bytes;
} okv_row_array;

typedef struct okv_pages {
  int32_t n_layers, page_tokens;           /* T: a power of two in [1, 1024]                          */
  int32_t max_seqs, max_pages_per_seq;     /* max_pages_per_seq * T below 2^31                        */
  int32_t n_pages;
  int32_t n_arrays, n_rows;                /* used entries of the next two                            */
  okv_page_array arrays[OKV_PAGES_MAX_ARRAYS];
  okv_row_array rows[OKV_PAGES_MAX_ROWS];
  int32_t *table, *lens, *refs, *status;
  void *workspace;                         /* okv_pages_workspace_bytes(n_pages), 16-byte aligned     */
  int64_t workspace_bytes;
} okv_pages;

int64_t okv_pages_workspace_bytes(int32_t n_pages);

/* Sequence seqs[i] grows by n_new[i] >= 0 tokens: takes the pages that it lacks and raises lens.  Nothing is done
 * while status[0] and status[3] both hold a code.
 *   seqs [n] distinct, or NULL: i;  n_new [n], or NULL: 1 each */
int okv_pages_extend(const okv_pages *p, int32_t n, const int32_t *seqs, const int32_t *n_new, void *stream);

/* Sequence dst[i], which must be empty, becomes a fork of src[i]: shares its full pages and copies the
 * rest.  src [n] (a sequence may be forked several times), dst [n] distinct.  A src that is empty gives
 * an empty fork. */
int okv_pages_fork(const okv_pages *p, int32_t n, const int32_t *src, const int32_t *dst, void *stream);

/* The sequences become empty; pages that belong to no other are free.  seqs [n] (twice the same: once). */
int okv_pages_free(const okv_pages *p, int32_t n, const int32_t *seqs, void *stream);

/* Sequence seqs[i] loses its last n_drop[i] >= 0 tokens (drafted ones that were rejected); pages that no token of it is in any longer
 * belong to it no more.  Nothing is done while status[0] and status[3] both hold a code (the tokens that are to go
 * were never added).  OKV_ESTATE, and nothing changes, where a sequence has fewer tokens, where the page that its new last token leaves partly
 * filled is shared (a shared page is full), and where a row array no longer holds the rows of a group that becomes partly filled (with rows = 32: the
 * new length is no multiple of 32 and lies below the last one that the old length has passed).
 *   seqs [n] distinct, or NULL: i;  n_drop [n] */
int okv_pages_shrink(const okv_pages *p, int32_t n, const int32_t *seqs, const int32_t *n_drop, void *stream);

/* Moves pages so that the pages in use are 0 .. n_used - 1: the m-th of those with ids from n_used on goes
 * to the m-th free id below.  Table and refs follow.  Pages keep what they hold until they are taken
 * again. */
int okv_pages_compact(const okv_pages *p, void *stream);

/* Copies pages src_ids[i] of p's arrays to pages dst_ids[i] of the arrays `to` (HOST array of p->n_arrays
 * entries with the same page_bytes, of to_pages pages): gathering what is to be moved to the host in one
 * copy, scattering what came back, copying within a pool.  No page may be both read and written, none be written twice.
 * Neither table nor refs are looked at. */
int okv_pages_copy(const okv_pages *p, int32_t n, const int32_t *src_ids, const int32_t *dst_ids,
                   const okv_page_array *to, int32_t to_pages, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* OKV_PAGES_H */
