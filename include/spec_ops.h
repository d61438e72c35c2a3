/*
 * Operators on caller buffers that a layer of a checkpoint with 8-bit floating point weights (e4m3, one scale per
 * 128 x 128 block) and normed query / key heads needs: the row quantiser, the product, and the heads' norm and
 * rotation.  The layers of the engine of spec.h do the last one's arithmetic after spec_set_qk_norm(), in a kernel of
 * their own that reads the projection's result and writes the queries and the cache; the first two they do not use.
 *
 * Same conventions as spec.h: 0 or a negative SPEC_E* code, the text of a failure from spec_last_error(NULL); "device"
 * pointers belong to the current device; work is enqueued on `stream` (a hipStream_t, NULL: the null stream), nothing
 * synchronises or allocates, and every call may be captured into a graph (kernel launches only).  The library keeps no
 * state between calls: calls on different streams may overlap as long as their outputs and workspaces differ.  Inputs,
 * outputs and workspaces must not overlap unless stated otherwise.  R == 0 is a call without work; R is at most 2^30, and
 * R * ceil(K / 128) stays below 2^31.
 */
#ifndef SPEC_OPS_H
#define SPEC_OPS_H

#include <stdint.h>

#include "spec.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of the operators below besides SPEC_F32 and SPEC_BF16: e4m3 (sign, 4 exponent bits of bias 7, 3
 * fraction bits, largest value 448, no infinities).  Not a storage type of spec_shape. */
enum { SPEC_F8 = 3 };

/* Quantise rows: per row and block of 128 columns (the last one may be shorter)
 *     a = max(max |x|, 2^-96),  scale = a / 448,  q = e4m3(x * (448 / a)),
 * quotients and product in fp32, each rounded to nearest even.  x: device, dtype SPEC_F32 or SPEC_BF16, row r at
 * element r * ldx (ldx >= K), any alignment of its element type; q: device e4m3 [R][K], 16-byte aligned; scale: device
 * fp32 [ceil(K / 128)][R] (the product reads the scales of a block of columns together).  16 <= K <= 2^22, K % 16 == 0.
 * A NaN stays a NaN in its place; a block with an infinity gets an infinite scale, and products over it are NaN. */
int spec_k_quant_f8(const void *x, int32_t dtype, int64_t ldx, int32_t R, int32_t K, void *q, float *scale, void *stream);

/* y[r][n] = sum over blocks b of x_scale[b][r] * w_scale[n / 128][b] * sum over k in block b of x[r][k] * w[n][k].
 * w: device e4m3 [N][K] row-major as a checkpoint holds it, 16-byte aligned; w_scale: device fp32 [ceil(N / 128)]
 * [ceil(K / 128)]; 1 <= N <= 2^30, 16 <= K <= 2^22, K % 16 == 0.  y: device, y_dtype SPEC_F32 or SPEC_BF16, row r at
 * element r * ldy (ldy >= N); columns N .. ldy - 1 are left alone.
 * Sums are held in fp32.  With y_dtype SPEC_F32 the products enter them whole: a result is off by at most (131 + ceil(K / 128))
 * 2^-23 of the sum of its terms' magnitudes, and for terms of either sign by about 1e-7 of its typical size (the root of
 * the sum of the squared terms).  With SPEC_BF16 the matrix unit may sum eight neighbouring products at a time to 13 bits
 * below the largest of them: at most 7 * 2^-13 of the sum of the magnitudes, typically 2e-5 to 3e-5 of a result's size (its
 * rounding to bf16: 2e-3 of its value).  A caller who needs whole sums in bf16 takes SPEC_F32 results and rounds them.
 * The same call gives the same bits every time.  How the sums are formed (their order and, for SPEC_BF16, which of them are
 * whole) depends on R, N, K, the types, the alignment and stride of x and the size of the workspace, so a row's last bits
 * may differ between calls that differ in these.
 * The product of two scales is an fp32 number: where it leaves fp32's normal range, so does the precision (beyond 2^128
 * the results are infinities or NaN).
 *  - x_dtype SPEC_F8: x e4m3 [R][K] (ldx == K), 16-byte aligned, with x_scale device fp32 [ceil(K / 128)][R], both as
 *    spec_k_quant_f8 leaves them.
 *  - x_dtype SPEC_F32 / SPEC_BF16: rows as for spec_k_quant_f8, quantised by the call by its rule; x_scale NULL.
 * workspace: device scratch, 16-byte aligned, of at least spec_k_gemm_f8_workspace() bytes (0: NULL will do).  More
 * lets products with few output columns share K out over workgroups; from 32 MiB beyond that on, the result no longer
 * depends on its size.  Contents need no preparation and are overwritten; calls that may overlap (captured graphs replayed
 * on two streams included) need workspaces of their own.  SPEC_EINVAL when it is too small. */
int spec_k_gemm_f8(const void *w, const float *w_scale, int32_t N, int32_t K, const void *x, int32_t x_dtype, int64_t ldx,
                   const float *x_scale, int32_t R, void *y, int32_t y_dtype, int64_t ldy, void *workspace,
                   int64_t workspace_bytes, void *stream);

/* Bytes of workspace spec_k_gemm_f8 must be given: the quantised rows, 132 * R * ceil(K / 128), for fp32 / bf16 rows,
 * 0 for e4m3 rows; SPEC_EINVAL for sizes the product refuses. */
int64_t spec_k_gemm_f8_workspace(int32_t K, int32_t R, int32_t x_dtype);

/* RMS norm of each query and key head, then the rotation of spec.h (element j pairs with j + hd / 2), in one pass:
 *     h <- h / sqrt(mean(h^2) + eps) * norm,   (h[j], h[j + hd/2]) <- (h[j] c - h[j + hd/2] s, h[j + hd/2] c + h[j] s)
 * with c = rope_cos[pos[r]][j], s = rope_sin[pos[r]][j], in fp32.  So are the squares: elements beyond 2^59 overflow them,
 * and where eps is 0 (it may be) heads with nothing above 2^-60 lose them; a head of zeros is then NaN.
 * q, k: device, dtype SPEC_F32 or SPEC_BF16, head i of row r at element r * ldq + i * hd (k likewise with ldk): the query
 * and key columns of a fused QKV row, or arrays of their own; ldq >= nq * hd, ldk >= nkv * hd.  q_norm, k_norm: device
 * fp32 [hd].  rope_cos, rope_sin: device fp32 [n_pos][hd / 2].  pos: device int32 [R]; a row whose position lies outside
 * 0 .. n_pos - 1 (padding) is left as it was in the outputs.  q_out, k_out: device, out_dtype, strides ldqo, ldko; they
 * may be the inputs themselves (same pointer, type and stride).  hd even, 2 <= hd <= 512; nq, nkv >= 0, not both 0 (the
 * pointers of the one that is 0 are ignored); R * (nq + nkv) < 2^31. */
int spec_k_qk_norm_rope(const void *q, int64_t ldq, int32_t nq, const void *k, int64_t ldk, int32_t nkv, int32_t dtype,
                        int32_t hd, int32_t R, const float *q_norm, const float *k_norm, float eps, const float *rope_cos,
                        const float *rope_sin, int32_t n_pos, const int32_t *pos, void *q_out, int64_t ldqo, void *k_out,
                        int64_t ldko, int32_t out_dtype, void *stream);

#ifdef __cplusplus
}
#endif
#endif
