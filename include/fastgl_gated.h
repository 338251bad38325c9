/*
 * fastgl_gated.h - C ABI of the gated feed-forward update on MI355X (gfx950): what
 * a deep sampled GNN puts in the place of act(H W + b) (paper Section 2.1, Eq. 2,
 * leaves Update abstract).
 *
 *   forward   G = X Wg + bg,  U = X Wu + bu,  P = act(G) * U
 *   backward  dG = dP * U * act'(G),  dU = dP * act(G)
 *             dX = dG Wg^T + dU Wu^T,  dWg = X^T dG,  dWu = X^T dU
 *             dbg, dbu = column sums of dG, dU
 *
 * act: SiLU g s(g) with s(g) = 1 / (1 + exp(-g)); GELU g (1 + erf(g / sqrt 2)) / 2; ReLU;
 * sigmoid s(g).  X [M,K], Wg, Wu [K,N], G, U, P, dP [M,N]: dense row-major without
 * padding, fp32 or (bit patterns in uint16_t) bf16, all of one dtype; biases and their
 * gradients fp32 [N].  The weight gradients are of the weights' dtype: with bf16 their terms
 * dG, dU are already rounded to bf16, so that more bits would hold little.
 *
 * Both products of a pass share one kernel.  They run on the bf16 matrix cores with fp32
 * accumulation; fp32 elements are cut into three bf16 pieces whose sum is the element
 * exactly, and six of the nine piece products are added, smallest first (relative error of a
 * product at most 2^-23).  Few rows are multiplied with plain fp32 multiply-adds.  bf16
 * results are rounded once, from fp32.  dG and dU, formed in fp32, are rounded to bf16 on their way to bf16
 * products, at every size (fastgl_gated_bwd_fine: to two bf16 pieces, within 2^-17); their column sums are formed
 * before that.  Elements that are not finite: every sum such an
 * element enters is not finite, and no other changes (from fp32 pieces it is NaN, also for
 * finite elements above 3.39e38); act of an infinite G is what IEEE arithmetic makes of the formula.
 *
 * act(G) from G, before it is rounded to its type, is within 20 x 2^-24 of itself for GELU (bf16: another
 * 4e-5 + g^2 2^-23), (8 + 2 |g|) x 2^-24 for SiLU and the sigmoid, also far below 0 (values below 2^-119 may be 0).
 *
 * Conventions are those of fastgl_agg.h: caller-owned DEVICE memory aligned to the element
 * size; nothing is allocated, scratch comes from `workspace` (256-byte aligned); work is enqueued
 * on `stream` without synchronising the host; outputs are overwritten in full and must not
 * overlap inputs or each other; results do not depend on scheduling.  0 <= M < 2^31-1-1024,
 * 0 <= K, N <= 2^20; K == 0 gives G = bg, U = bu; M == 0 or N == 0 write what is left
 * (zeros where a sum has no terms).
 */
#ifndef FASTGL_GATED_H
#define FASTGL_GATED_H

#include "fastgl_agg.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { FASTGL_ACT_SILU = 0, FASTGL_ACT_GELU = 1, FASTGL_ACT_RELU = 2, FASTGL_ACT_SIGMOID = 3 } fastgl_act;

/* Bytes of workspace of a call: packed operands (fp32 pieces; rows that are no multiple of 16
 * bytes), dG and dU, partial sums.  `aligned`: whether X, Wg and Wu start at multiples of 16 bytes;
 * 0 is the bound for both.  The forward call may need none. */
size_t fastgl_gated_fwd_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned);
size_t fastgl_gated_bwd_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned);
size_t fastgl_gated_bwd_fine_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned);

/* Forward pass.  bg, bu may be NULL; G and U, kept for the backward pass, may be NULL. */
fastgl_status fastgl_gated_fwd(fastgl_dtype dtype, const void *X, const void *Wg, const void *Wu, const float *bg,
                               const float *bu, int64_t M, int64_t K, int64_t N, fastgl_act act, void *P, void *G, void *U,
                               void *workspace, size_t workspace_bytes, void *stream);

/* Backward pass from G and U as the forward pass wrote them.  Any of dX, dWg, dWu, dbg, dbu may
 * be NULL; X is read for dWg and dWu alone, Wg and Wu for dX alone. */
fastgl_status fastgl_gated_bwd(fastgl_dtype dtype, const void *X, const void *Wg, const void *Wu, const void *G,
                               const void *U, const void *dP, int64_t M, int64_t K, int64_t N, fastgl_act act, void *dX,
                               void *dWg, void *dWu, float *dbg, float *dbu, void *workspace, size_t workspace_bytes,
                               void *stream);

/* The same with dG and dU in two bf16 pieces where the type is bf16: what is left of their rounding is below the
 * results' own, for twice the products.  fp32: the same call. */
fastgl_status fastgl_gated_bwd_fine(fastgl_dtype dtype, const void *X, const void *Wg, const void *Wu, const void *G,
                                    const void *U, const void *dP, int64_t M, int64_t K, int64_t N, fastgl_act act, void *dX,
                                    void *dWg, void *dWu, float *dbg, float *dbu, void *workspace, size_t workspace_bytes,
                                    void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FASTGL_GATED_H */
