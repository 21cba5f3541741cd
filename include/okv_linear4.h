/*
 * okv_linear4 -- the linear layers of okv_layer.h with 4-bit weights, for one MI355X.
 *
 * In the decode stage every weight is read once per step (paper §IV-D: 8 h1^2 + 4 h1 h2 flops per token and
 * layer, a few dozen tokens): the products are bound by the bytes of the weights, a quarter of fp16's here.
 *
 *     W[n][k] = (code[n][k] - zero[n][k / group]) * scale[n][k / group]
 *
 * code in 0 .. 15; scale fp16; zero in 0 .. 15, or 8 everywhere.  The products take code - zero exactly in
 * fp16 on the matrix cores and multiply the fp32 sums of a group by its scale: weights are not rounded again.
 *
 * Faster than the fp16 products of okv_layer.h for few rows; for many they save memory and cost time.  us, codes and weights from HBM, groups of
 * 128 / of 32 / fp16, 16384 x 4096: 16 rows 11.3 / 12.2 / 25.0, 64 rows 23.4 / 28.4 / 25.1, 128 rows 32 / 50 / 33, 256 rows 62 / 96 / 47, 1024
 * rows 239 / 370 / 115, 4096 rows 945 / 1453 / 461; 4096 x 4096: 32 rows 9.8 / 10.1 / 9.7, 256 rows 23.8 / 27.5 / 19.1, 1024 rows 63 / 95 / 39.
 *
 * Conventions as in okv_layer.h.
 */
#ifndef OKV_LINEAR4_H
#define OKV_LINEAR4_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define OKV_LINEAR4_MAX_BATCH 4096   /* rows per call                                                 */

/* Bytes of a packed matrix: n_out a multiple of 16, n_in a multiple of 32 and of group, group 32, 64 or 128.
 * Codes first: blocks of 16 features x 128 inputs (the last block's inputs padded), as the 64 x 16 bytes that a
 * wavefront loads with one instruction: 32-bit word j of lane l holds inputs 32 j + 8 (l / 16) .. + 7 of feature l % 16, input 2 p
 * of them in bits 4 p .. 4 p + 3 and input 2 p + 1 in bits 16 + 4 p .. 19 + 4 p.  Then the scales, fp16
 * [n_out / 16][blocks][4][128 / group][4] (feature 4 i + j of the 16 at [..][i][..][j]), and, with zeros, the zeros, bytes
 * [n_out / 16][blocks][16][128 / group]. */
int64_t okv_linear4_packed_bytes(int32_t n_out, int32_t n_in, int32_t group, int32_t zeros);

/* Packs a matrix that is quantised already.
 *   dst     okv_linear4_packed_bytes bytes
 *   codes   [n_out][n_in / per_byte] bytes, row-major: one code a byte (per_byte 1), or two, the even input in the low
 *           half (per_byte 2)
 *   scales  fp16 [n_out][n_in / group];  zeros  bytes of that shape, or NULL */
int okv_linear4_pack(void *dst, const void *codes, int32_t per_byte, const void *scales, const void *zeros,
                     int32_t n_out, int32_t n_in, int32_t group, void *stream);

/* Quantises fp16 weights src [n_out][n_in] row-major and packs them.  Every group by itself, in fp32:
 *   zeros 0:  scale = max |w| / 7,                           code = clamp(rne(w / scale) + 8, 0, 15)
 *   zeros 1:  scale = (max(w, 0) - min(w, 0)) / 15,  zero = rne(-min(w, 0) / scale),
 *             code = clamp(rne(w / scale) + zero, 0, 15)
 * with the scale rounded to fp16 before it is divided by (a group whose scale is 0 in fp16 has scale 0).
 * A group with a weight that is infinite or NaN has scale NaN, so that every result of its feature is NaN. */
int okv_linear4_quantize(void *dst, const void *src, int32_t n_out, int32_t n_in, int32_t group, int32_t zeros, void *stream);

/* out = act(x W^T + bias) + residual, as okv_linear.
 *   x         fp16 [m][n_in], m <= OKV_LINEAR4_MAX_BATCH; must not overlap out
 *   packed    as the calls above leave it, with the same n_out, n_in, group and zeros
 *   bias      fp16 [n_out] or NULL;  residual  fp16 [m][n_out] or NULL (n_seg must be 1; may be out[0])
 *   out       HOST array of n_seg (1 to 3) DEVICE pointers: run s of the output features is written as fp16
 *             [m][cols[s]] to out[s]
 *   cols      HOST [n_seg] multiples of 16 that add up to n_out, or NULL: equal runs
 *   relu      1: act = max(., 0), NaN where the argument is (okv_linear gives 0 there)
 *   workspace okv_linear4_workspace_bytes bytes of scratch, 16-byte aligned; with less (or NULL) a form that needs none runs.
 *             Calls that may run at the same time need workspaces of their own. */
int okv_linear4(const void *x, const void *packed, const void *bias, const void *residual, void *const *out,
                const int32_t *cols, int32_t n_seg, int32_t m, int32_t n_out, int32_t n_in, int32_t group,
                int32_t zeros, int32_t relu, void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of workspace that okv_linear4 wants for this shape (0: none); < 0 on a bad shape. */
int64_t okv_linear4_workspace_bytes(int32_t m, int32_t n_out, int32_t n_in);

#ifdef __cplusplus
}
#endif
#endif /* OKV_LINEAR4_H */
