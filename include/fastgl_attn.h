/*
 * fastgl_attn.h - C ABI of attention over the sampled neighbours of a block on
 * MI355X (gfx950): the layer of a graph transformer, dot products of a target's
 * query with its neighbours' keys in the place of the edge weights of Eq. 1 (paper
 * Section 2.1), several heads in one call and no array per edge and head in memory.
 *
 *   forward   s_e    = scale * <Q[u,h,:], K[v_e,h',:]> + bias[bucket_e, h]       e an edge of row u, h' = h / (heads / kv_heads)
 *             lse_u  = log sum over row u of exp(s_e)
 *             O[u,h] = sum over row u of p_e V[v_e,h',:],   p_e = exp(s_e - lse_u)
 *   backward  dp_e = <dO[u,h,:], V[v_e,h',:]>,  ds_e = p_e (dp_e - sum over row u of p dp)
 *             dQ[u,h] = scale * sum over row u of ds_e K[v_e,h',:]
 *             dK[v,h'] = scale * sum over the edges of source v and the heads h of h' of ds_e Q[u_e,h,:],
 *             dV[v,h'] = sum over the same of p_e dO[u_e,h,:]
 *             dbias[b,h] = sum over the edges of bucket b of ds_e
 *   The probabilities are computed again from Q, K and the bias: neither O nor lse nor an array of
 *   edges has to be kept between the passes.
 *
 * Blocks are the CSR-by-destination blocks of fastgl_agg.h.  Q, O and their gradients are
 * [num_dst, heads * width], K, V and theirs [num_src, kv_heads * width]; fp32, or bf16 (bit
 * patterns in uint16_t), all of one dtype.  Rows may lie further apart than they are long (the ld
 * arguments, in elements): Q, K and V may be columns of one projection's output, and dQ, dK and dV columns
 * of its gradient; what lies between rows is neither read nor written.  lse is fp32 [num_dst, heads], bias and
 * dbias fp32 [num_buckets, heads].
 *
 * bucket int32 [num_edges], in edge order: relation, distance in time or hops, or whatever else
 * the learned bias goes by.  An edge whose bucket is negative, or num_buckets and above, is left
 * out of the attention: it adds nothing anywhere, whatever its neighbour's row holds.  Without a
 * bias (NULL) buckets may be given all the same, to leave edges out (the negative ones; num_buckets is
 * not read).  An edge whose bias or score is -inf adds nothing either.  A row that no
 * edge is left of has O = 0, lse = -inf, dQ = 0.
 *
 * Products and sums are fp32 (bf16 inputs are exact in it), sums of a row in runs of edges (long rows: in chunks of
 * fastgl_long_row_chunk()) joined in a fixed order, dbias in fp32 within a workgroup and fp64 over them; results are
 * rounded once.  Results do not depend on scheduling.  NaN in a row gives NaN where it takes part and changes no other row of O
 * and dQ; so may infinities in Q, K and dO, and infinities in V, where IEEE arithmetic would give a score or a weight that is not NaN.
 *
 * Conventions are those of fastgl_agg.h: caller-owned DEVICE memory, aligned to the element size;
 * nothing is allocated, scratch comes from `workspace` (256-byte aligned); work is enqueued on
 * `stream` without synchronising the host; outputs are overwritten in full and must not overlap inputs or each other
 * (interleaved columns do not overlap); calls that share a workspace must be ordered.  1 <= width <= 256,
 * kv_heads >= 1 divides heads, heads <= 4096, heads * width <= 65536, 1 <= num_buckets <= 65536 with a bias.
 */
#ifndef FASTGL_ATTN_H
#define FASTGL_ATTN_H

#include "fastgl_agg.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What both passes read (host struct; the pointers inside are device pointers). */
typedef struct {
    const int32_t *indptr, *indices;
    int64_t num_dst, num_src, num_edges;
    const int32_t *bucket;              /* [num_edges] or NULL */
    const float *bias;                  /* [num_buckets, heads] or NULL; needs bucket */
    int64_t num_buckets;
    int64_t heads, kv_heads, width;
    float scale;
    fastgl_dtype dtype;
    const void *Q, *K, *V;
    int64_t ldq, ldk, ldv;              /* elements between rows */
} fastgl_attn_desc;

/* Bytes of workspace of a call; of *desc, sizes and dtype are read, and whether bucket and bias are NULL.  Room for the bookkeeping is
 * in it, so that plan == NULL works.  0 where the sizes are refused. */
size_t fastgl_attn_workspace_bytes(const fastgl_attn_desc *desc, int backward);

/* Forward pass.  lse may be NULL.  plan: NULL, or a plan of exactly this block with
 * FASTGL_PLAN_FWD; it is read for rows of more than fastgl_long_row_threshold() edges, and a block of so few edges needs
 * none.  With NULL the bookkeeping is rebuilt inside `workspace`.  With FASTGL_PLAN_SHORT_DST_ROWS every row of a block
 * of at most 2^24 edges is walked by one wavefront. */
fastgl_status fastgl_attn_fwd(const fastgl_attn_desc *desc, void *O, int64_t ldo, float *lse, const fastgl_plan *plan,
                              void *workspace, size_t workspace_bytes, void *stream);

/* Backward pass.  Any of dQ, dK, dV and dbias may be NULL.  plan: NULL, or a plan with
 * FASTGL_PLAN_ALL, and FASTGL_PLAN_PERM as well where buckets are given. */
fastgl_status fastgl_attn_bwd(const fastgl_attn_desc *desc, const void *dO, int64_t lddo, void *dQ, int64_t lddq,
                              void *dK, int64_t lddk, void *dV, int64_t lddv, float *dbias, const fastgl_plan *plan,
                              void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FASTGL_ATTN_H */
