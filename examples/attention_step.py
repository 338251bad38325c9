"""A training step of a graph transformer's layer on a sampled block: how attention over the sampled neighbours and the
classifier's loss are used with the calls around them.

    forward   q, k, v = X Wq, X Wkv                          k and v side by side in one product
              A = attention(q[:targets], k, v, bias)         softmax over the sampled neighbours, a bias for each relation
              n, s = norm(X[:targets] + A Wo)                one call; s would be the next layer's residual
              loss = cross entropy(n Wc + bc, labels)        the class scores are not kept
    backward  the same chain from its end: no array of edges and heads and no class scores exist anywhere

Edges of relation -1 take no part (an edge to the label's own node, a padded one), nodes of label -1 have no loss.

Run `python examples/attention_step.py` on an MI355X: a few training steps on a synthetic block.
"""
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2409_14939_amd import binding as B

EPS = 1e-6


def make_params(width, heads, kv_heads, head, relations, classes, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)

    def matrix(k, n):
        return (torch.randn(k, n, generator=g) / k ** 0.5).to(dtype).cuda()
    return dict(Wq=matrix(width, heads * head), Wkv=matrix(width, 2 * kv_heads * head), bias=torch.zeros(relations, heads).cuda(),
                Wo=matrix(heads * head, width), w=torch.ones(width).cuda(), Wc=matrix(width, classes), bc=torch.zeros(classes).cuda())


def split(kv):
    half = kv.shape[1] // 2
    return kv[:, :half], kv[:, half:]


def forward(p, block, relation, X, labels, heads, kv_heads):
    """(loss of every target, what the backward pass needs); block = (indptr, indices, plan)."""
    indptr, indices, plan = block
    targets = X[:indptr.numel() - 1]
    q, kv = B.fastgl_update_fwd(targets, p["Wq"], None, False), B.fastgl_update_fwd(X, p["Wkv"], None, False)
    A, _ = B.fastgl_attn_fwd(indptr, indices, q, *split(kv), heads, kv_heads, bucket=relation, bias=p["bias"], want_lse=False, plan=plan)
    n, s, rstd = B.fastgl_norm_fwd(B.fastgl_update_fwd(A, p["Wo"], None, False), p["w"], EPS, residual=targets)
    loss, lse = B.fastgl_loss_fwd(n, p["Wc"], p["bc"], labels)
    return loss, dict(q=q, kv=kv, A=A, n=n, s=s, rstd=rstd, lse=lse)


def backward(p, block, relation, X, labels, kept, dloss, heads, kv_heads):
    """Gradients of the parameters and of X."""
    indptr, indices, plan = block
    num_dst = indptr.numel() - 1
    k, g = kept, {}
    dn, g["Wc"], g["bc"] = B.fastgl_loss_bwd(k["n"], p["Wc"], p["bc"], labels, k["lse"], dloss)
    dD, ds, g["w"] = B.fastgl_norm_bwd(k["s"], p["w"], k["rstd"], dn)
    dA, g["Wo"], _ = B.fastgl_update_bwd(k["A"], p["Wo"], None, dD, False, want=("dH", "dW"))
    dkv = torch.empty_like(k["kv"])                      # dK and dV side by side, as the projection's gradient wants them
    dK, dV = split(dkv)
    dq, _, _, g["bias"] = B.fastgl_attn_bwd(indptr, indices, k["q"], *split(k["kv"]), dA, heads, kv_heads, bucket=relation, bias=p["bias"],
                                            dK=dK, dV=dV, plan=plan)
    dT, g["Wq"], _ = B.fastgl_update_bwd(X[:num_dst], p["Wq"], None, dq, False, want=("dH", "dW"))
    dX, g["Wkv"], _ = B.fastgl_update_bwd(X, p["Wkv"], None, dkv, False, want=("dH", "dW"))
    dX[:num_dst] += dT
    dX[:num_dst] += ds
    return g, dX


def main():
    import blockgen as bg
    blk = bg.make_config(1).blocks[0]
    indptr, indices = torch.from_numpy(blk.indptr).cuda(), torch.from_numpy(blk.indices).cuda()
    plan = B.fastgl_block_plan_create(indptr, indices, blk.num_src, B.PLAN_ALL | B.PLAN_PERM)
    heads, kv_heads, head, width, relations, classes = 8, 2, 16, 64, 5, 47
    g = torch.Generator().manual_seed(0)
    X = torch.randn(blk.num_src, width, generator=g).bfloat16().cuda()
    relation = torch.randint(-1, relations, (blk.num_edges,), generator=g, dtype=torch.int32).cuda()
    labels = torch.randint(-1, classes, (blk.num_dst,), generator=g).cuda()
    p = make_params(width, heads, kv_heads, head, relations, classes, torch.bfloat16)
    dloss = torch.full((blk.num_dst,), 1.0 / max(int((labels >= 0).sum()), 1), device="cuda")
    for step in range(5):
        loss, kept = forward(p, (indptr, indices, plan), relation, X, labels, heads, kv_heads)
        grads, _ = backward(p, (indptr, indices, plan), relation, X, labels, kept, dloss, heads, kv_heads)
        print(f"step {step}: mean loss {(loss * dloss).sum().item():.4f}", flush=True)
        for name, grad in grads.items():
            p[name] -= 0.1 * grad.to(p[name].dtype)


if __name__ == "__main__":
    main()
