/*
 * fastgl_loss.h - C ABI of a classifier's loss on MI355X (gfx950): softmax cross
 * entropy of the class scores of a mini-batch's target nodes, which an update phase
 * without an activation gives (paper Section 2.1, Eq. 2), from the rows and weights
 * themselves.  The scores are formed tile by tile and never kept: their number, rows
 * times classes, bounds neither pass.
 *
 *   forward   z = H W + b,  lse[i] = log sum_n exp z[i,n],  loss[i] = lse[i] - z[i, label[i]]
 *   backward  dZ[i,n] = g[i] (exp(z[i,n] - lse[i]) - [n == label[i]])      g = dloss, the gradient of loss
 *             dH = dZ W^T,  dW = H^T dZ,  db = column sums of dZ
 *
 * H [M,K], W [K,N], dH, dW: dense row-major without padding, fp32 or (bit patterns in
 * uint16_t) bf16, all of one dtype; b, db [N], loss, lse, dloss [M] fp32; label int64 [M].  A row with a
 * negative label has no loss: loss 0, dH 0, nothing added to dW and db, whatever H and dloss hold there (lse is
 * that of its scores).  A label of N and above gives NaN: the row's loss and dH, and dW and db.
 *
 * Scores are formed on the bf16 matrix cores with fp32 accumulation, from three bf16 pieces of each fp32 element (six of nine
 * piece products, relative error of a product at most 2^-23), or, in small calls, as fp32 multiply-adds.  Maxima and sums are fp32
 * within a tile and over tiles.  dZ, formed in fp32, goes into the two products within 2^-17 of itself in bf16 calls (two bf16 pieces) and within
 * 2^-24 in fp32 ones (three), or as it is (small calls).  fastgl_loss_bwd_coarse rounds it to one bf16 in bf16 calls, at every size: dH and dW are
 * up to sqrt 2 times as far off, for half the products; fp32 calls are as with fastgl_loss_bwd.  db is of the unrounded values.  Results are rounded once.  exp(z - lse) is
 * off by 2^-23 (2 + |z| + |lse|) of itself and by its score's error.  A row with a score of NaN or +inf has loss and dH NaN; scores of
 * -inf and of the type's lowest value (a bias that rules a class out) weigh nothing where another class remains.  The pieces of an infinite
 * fp32 element of H or W are not finite either: its scores are NaN (in small calls what IEEE arithmetic gives).
 *
 * Conventions are those of fastgl_agg.h: caller-owned DEVICE memory aligned to the element size; nothing is
 * allocated, scratch comes from `workspace` (256-byte aligned); work is enqueued on `stream` without synchronising the host;
 * outputs are overwritten in full and must not overlap inputs or each other; results do not depend on scheduling.
 * 0 <= M < 2^31-1-1024, 0 <= K <= 2^20, 1 <= N <= 2^21 where M > 0.
 */
#ifndef FASTGL_LOSS_H
#define FASTGL_LOSS_H

#include "fastgl_agg.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of workspace of a call.  `aligned`: whether H and W start at multiples of 16 bytes; 0 is the bound for both.  The classes are
 * taken in pieces, so that the forward pass's statistics, the backward pass's dZ and packed weights stay below 1 GiB each (256 classes at least). */
size_t fastgl_loss_fwd_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned);
size_t fastgl_loss_bwd_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned);
size_t fastgl_loss_bwd_coarse_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned);

/* Forward pass.  b may be NULL; lse, which the backward pass reads, may be NULL. */
fastgl_status fastgl_loss_fwd(fastgl_dtype dtype, const void *H, const void *W, const float *b, const int64_t *label, int64_t M,
                              int64_t K, int64_t N, float *loss, float *lse, void *workspace, size_t workspace_bytes, void *stream);

/* Backward pass from lse as the forward pass wrote it.  Any of dH, dW, db may be NULL. */
fastgl_status fastgl_loss_bwd(fastgl_dtype dtype, const void *H, const void *W, const float *b, const int64_t *label,
                              const float *lse, const float *dloss, int64_t M, int64_t K, int64_t N, void *dH, void *dW, float *db,
                              void *workspace, size_t workspace_bytes, void *stream);

/* The same with dZ rounded to one bf16 for the products of bf16 calls. */
fastgl_status fastgl_loss_bwd_coarse(fastgl_dtype dtype, const void *H, const void *W, const float *b, const int64_t *label,
                                     const float *lse, const float *dloss, int64_t M, int64_t K, int64_t N, void *dH, void *dW, float *db,
                                     void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FASTGL_LOSS_H */
