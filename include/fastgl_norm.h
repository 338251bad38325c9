/*
 * fastgl_norm.h - C ABI of what stands between the aggregations of a deep
 * (residual) sampled GNN on MI355X (gfx950): root-mean-square norm with the
 * residual's addition, dropout from a counter-based generator, and rows held in
 * 8 bits.
 *
 *   h    = R + drop(X)                      (either part may be absent)
 *   rstd = 1 / sqrt(mean over the row of h^2 + eps)
 *   Y    = h * rstd * w
 *   drop(x)[i,j] = x[i,j] * 65536 / (65536 - t) where keep(i,j), else 0;
 *                  t = round(65536 p), 0 <= p <= 1; the factor is rounded to fp32 first
 *   keep(i,j): half word j % 8 of Philox4x32-10(key = seed, counter =
 *                  (j / 8, i, offset)) is >= t; low half words first
 *
 * Row i of the mask is the same whatever the number of rows and columns.  What is
 * dropped is 0 also where it was NaN or infinite.  `rng` points to two int64 in
 * DEVICE memory, {seed, offset}: a captured graph reads them anew at every
 * replay, so a program advances the offset between two uses and passes the value
 * that the forward pass had to the backward pass; no mask is stored.  p == 0
 * needs no rng (it may be NULL).
 *
 * X, R, Y, S, dY and the like: [M, F] dense row-major fp32 or bf16 (bit patterns in
 * uint16_t), all of one dtype; w, rstd, dw and row scales are fp32.  Sums are
 * formed in fp32 within a row, over rows in fp32 and then fp64; h is normalised
 * before it is rounded; each result is rounded once (nearest even).  A row of zeros
 * gives zeros (eps > 0).  A row with an element that is not finite gives what IEEE
 * arithmetic gives and changes no other row (but dw).  Squares are summed in fp32:
 * a row whose squares exceed 3.4e38 has rstd = 0.
 *
 * Conventions are those of fastgl_agg.h: caller-owned DEVICE memory, aligned to
 * the element size; nothing is allocated; work is enqueued on `stream` without
 * synchronising the host; outputs are overwritten in full and must not overlap
 * inputs; what can be checked on the host is checked before any launch.
 * 0 <= M < 2^31-1-1024, 1 <= F <= 2^24.  Results do not depend on scheduling.
 */
#ifndef FASTGL_NORM_H
#define FASTGL_NORM_H

#include "fastgl_agg.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Forward pass.  R may be NULL (h = drop(X)); sum_out, where h is written for the
 * backward pass and the next residual, and rstd [M] may be NULL. */
fastgl_status fastgl_norm_fwd(fastgl_dtype dtype, const void *X, const void *R, const float *w, int64_t M, int64_t F,
                              float eps, const int64_t *rng, double p, void *sum_out, void *Y, float *rstd, void *stream);

/* The same with Y as e4m3 values (OCP, 448 the largest) and one scale a row:
 * scale[i] = max(max |Y[i,:]| / 448, 2^-126), Q the fp32 quotient Y / scale to the nearest, even.
 * NaN stays NaN and does not enter the maximum. */
fastgl_status fastgl_norm_fwd_e4m3(fastgl_dtype dtype, const void *X, const void *R, const float *w, int64_t M, int64_t F,
                                   float eps, const int64_t *rng, double p, void *sum_out, uint8_t *Q, float *scale,
                                   float *rstd, void *stream);

/* Bytes of workspace fastgl_norm_bwd needs where dw is asked for. */
size_t fastgl_norm_bwd_workspace_bytes(int64_t M, int64_t F);

/* Backward pass.  S is h as the forward pass wrote it (X where it had neither R nor
 * dropout), rstd what it wrote; dS (or NULL) is the gradient that reaches h from elsewhere
 * (the residual stream).
 *   n = S * rstd,  t = dY * w,  d = rstd * (t - n * mean(t * n)) + dS
 *   dR = d,  dX = drop(d) with the forward pass's rng and p,  dw = column sums of dY * n
 * Any of dX, dR, dw may be NULL; dw needs `workspace` (256-byte aligned). */
fastgl_status fastgl_norm_bwd(fastgl_dtype dtype, const void *S, const float *w, const float *rstd, const void *dY,
                              const void *dS, int64_t M, int64_t F, const int64_t *rng, double p, void *dX, void *dR,
                              float *dw, void *workspace, size_t workspace_bytes, void *stream);

/* Y = [R +] drop(X); R may be NULL.  The backward pass is the same call on dY without R. */
fastgl_status fastgl_dropout(fastgl_dtype dtype, const void *X, const void *R, int64_t M, int64_t F, const int64_t *rng,
                             double p, void *Y, void *stream);

/* Row gather from a table held in 8 bits: out[i,:] = scale[ids[i]] * table[ids[i],:], table e4m3
 * [table_rows, F], scale fp32 [table_rows], ids int64 [n], out [n, F] of `dtype`.  An ID outside the table
 * reads nothing and gives a row of NaN. */
fastgl_status fastgl_gather_rows_e4m3(const uint8_t *table, const float *scale, int64_t table_rows, const int64_t *ids,
                                      int64_t n, int64_t F, fastgl_dtype dtype, void *out, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FASTGL_NORM_H */
