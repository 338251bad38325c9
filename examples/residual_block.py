"""A residual gated layer on sampled blocks: how norm, dropout, the gated feed-forward update and 8-bit rows are used
next to the aggregation.

    forward   A = aggregate(X)                             mean over the sampled neighbours
              s = X[:targets] + drop(A),  n = norm(s)      one call; s is the residual stream
              P = silu(n Wg + bg) * (n Wu + bu)            one call
              D = P Wd + bd
              z = s + drop(D),  y = norm(z)                one call: the next norm adds the residual
              logits = y Wc + bc
    backward  the same chain from its end; no dropout mask exists anywhere: every use of the generator has an
              offset of its own, and the backward pass is given the one its forward pass had
    serving   y as e4m3 rows with a scale each: a feature table at a quarter of float32's bytes, gathered back by ID

Run `python examples/residual_block.py` on an MI355X: a few training steps on a synthetic block, then the table.
"""
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2409_14939_amd import binding as B

EPS = 1e-6


def make_params(width, hidden, classes, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)

    def matrix(k, n):
        return (torch.randn(k, n, generator=g) / k ** 0.5).to(dtype).cuda()
    return dict(w1=torch.ones(width).cuda(), Wg=matrix(width, hidden), Wu=matrix(width, hidden), bg=torch.zeros(hidden).cuda(),
                bu=torch.zeros(hidden).cuda(), Wd=matrix(hidden, width), bd=torch.zeros(width).cuda(), w2=torch.ones(width).cuda(),
                Wc=matrix(width, classes), bc=torch.zeros(classes).cuda())


def rng_states(seed, offset):
    """The generator's states of a step: one row {seed, offset} for each of its two dropouts."""
    return torch.tensor([[seed, offset], [seed, offset + 1]], dtype=torch.int64, device="cuda")


def forward(q, block, X, states, p):
    """(logits, what the backward pass needs); block = (indptr, indices, plan)."""
    indptr, indices, plan = block
    targets = indptr.numel() - 1
    A = B.fastgl_block_aggregate_fwd(indptr, indices, None, X.shape[0], "mean", X, plan=plan)
    n, s, rstd1 = B.fastgl_norm_fwd(A, q["w1"], EPS, residual=X[:targets], rng=states[0], p=p)
    P, G, U = B.fastgl_gated_fwd(n, q["Wg"], q["Wu"], q["bg"], q["bu"], "silu")
    D = B.fastgl_update_fwd(P, q["Wd"], q["bd"], False)
    y, z, rstd2 = B.fastgl_norm_fwd(D, q["w2"], EPS, residual=s, rng=states[1], p=p)
    logits = B.fastgl_update_fwd(y, q["Wc"], q["bc"], False)
    return logits, dict(n=n, s=s, rstd1=rstd1, P=P, G=G, U=U, y=y, z=z, rstd2=rstd2)


def backward(q, block, X, kept, dlogits, states, p):
    """Gradients of the parameters (weights of the dense products that fastgl_update_bwd gives: float32) and of X."""
    indptr, indices, plan = block
    k, g = kept, {}
    dy, g["Wc"], g["bc"] = B.fastgl_update_bwd(k["y"], q["Wc"], None, dlogits, False)
    dD, ds, g["w2"] = B.fastgl_norm_bwd(k["z"], q["w2"], k["rstd2"], dy, rng=states[1], p=p)
    dP, g["Wd"], g["bd"] = B.fastgl_update_bwd(k["P"], q["Wd"], None, dD, False)
    dn, g["Wg"], g["Wu"], g["bg"], g["bu"] = B.fastgl_gated_bwd(k["n"], q["Wg"], q["Wu"], k["G"], k["U"], dP, "silu")
    dA, dR, g["w1"] = B.fastgl_norm_bwd(k["s"], q["w1"], k["rstd1"], dn, dS=ds, rng=states[0], p=p)
    dX = B.fastgl_block_aggregate_bwd(indptr, indices, None, X.shape[0], "mean", dA, plan=plan)
    dX[:indptr.numel() - 1] += dR
    return g, dX


def table_of(q, kept):
    """The block's outputs as rows of a table held in 8 bits: (e4m3 rows, scales)."""
    Q, scale, _, _ = B.fastgl_norm_fwd_e4m3(kept["z"], q["w2"], EPS, want_rstd=False)
    return Q, scale


def main():
    import blockgen as bg
    import numpy as np

    blk = bg.make_config(1).blocks[0]
    ip, ix = torch.from_numpy(blk.indptr).cuda(), torch.from_numpy(blk.indices).cuda()
    block = (ip, ix, B.fastgl_block_plan_create(ip, ix, blk.num_src))
    width, hidden, classes, p = 64, 171, 10, 0.1
    rng = np.random.default_rng(0)
    X = torch.from_numpy(rng.standard_normal((blk.num_src, width)).astype(np.float32)).cuda()
    labels = torch.from_numpy(rng.integers(0, classes, blk.num_dst)).cuda()
    q = make_params(width, hidden, classes, torch.float32)
    for it in range(30):
        states = rng_states(seed=42, offset=2 * it)
        logits, kept = forward(q, block, X, states, p)
        prob = torch.softmax(logits, 1)
        loss = -torch.log(prob.gather(1, labels[:, None])).mean()
        dlogits = prob / blk.num_dst
        dlogits.scatter_add_(1, labels[:, None], torch.full((blk.num_dst, 1), -1.0 / blk.num_dst, device="cuda"))
        grads, _ = backward(q, block, X, kept, dlogits, states, p)
        for name, g in grads.items():
            q[name] -= 0.5 * g
        if it % 10 == 0 or it == 29:
            print(f"step {it:2d}  loss {loss.item():.4f}", flush=True)
    Q, scale = table_of(q, kept)
    ids = torch.randint(0, blk.num_dst, (1000,), device="cuda")
    rows = B.fastgl_gather_rows_e4m3(Q, scale, ids, "f32")
    off = (rows - kept["y"][ids]).norm() / kept["y"][ids].norm()
    print(f"table of {Q.shape[0]} rows in 8 bits; 1000 gathered rows are {off.item():.3f} off the float32 ones")


if __name__ == "__main__":
    main()
