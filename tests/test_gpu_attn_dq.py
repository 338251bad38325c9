"""dQ where the gradient of the weights is nearly the same over a row: rows of one edge, and values with a mean."""
import numpy as np
import pytest
import torch

import blockgen as bg
from attn_ref import U32, Attention
from gpu_util import dev_i32
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
HEADS = [(1, 1, 1), (2, 1, 3), (4, 4, 16), (6, 2, 20), (8, 8, 32), (4, 1, 47), (4, 2, 64), (3, 1, 200), (2, 2, 256)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads,kv,D", HEADS)
def test_a_row_of_one_edge_has_no_gradient(heads, kv, D, dtype):
    """One edge alone, one that is left of a row, at its start, its end and inside, of short rows and of chunks: the softmax is constant."""
    g = torch.Generator().manual_seed(D)
    degree = [1, 1, 2, 5, 16, 17, 40, 129, 256, 257, 700, 1300]
    ptr = np.concatenate([[0], np.cumsum(degree)]).astype(np.int32)
    sources = 60
    col = torch.randint(0, sources, (int(ptr[-1]),), generator=g).int()
    n, k = heads * D, kv * D
    make = lambda r, c: (3.0 + torch.randn(r, c, generator=g)).to(dtype).cuda()
    Q, K, V, dO = make(len(degree), n), make(sources, k), make(sources, k), make(len(degree), n)
    bias = torch.randn(2, heads, generator=g).cuda()
    for place in (0.0, 0.4, 1.0):
        bucket = torch.full((int(ptr[-1]),), -1, dtype=torch.int32)
        for i, d in enumerate(degree):
            bucket[int(ptr[i]) + int(place * (d - 1))] = i % 2
        O, lse = B.fastgl_attn_fwd(dev_i32(ptr), col.cuda(), Q, K, V, heads, kv, bucket=bucket.cuda(), bias=bias)
        dQ, dK, dV, dbias = B.fastgl_attn_bwd(dev_i32(ptr), col.cuda(), Q, K, V, dO, heads, kv, bucket=bucket.cuda(), bias=bias)
        assert bool(torch.isfinite(lse).all()) and bool(O.any()) and bool(dV.any())
        assert not bool(dQ.any()) and not bool(dK.any()) and not bool(dbias.any())


@pytest.mark.parametrize("heads,kv,D", [(1, 1, 3), (4, 2, 8), (3, 3, 20), (2, 1, 64)])
def test_values_with_a_mean(heads, kv, D):
    """dp are whole numbers of half a million that differ by some hundred: float32 holds them, and what they differ by is what dQ is of."""
    blk = bg.random_block(np.random.default_rng(D), 200, 300, 5.0, empty_frac=0.1, hub_rows=4, hub_deg=900)
    g = torch.Generator().manual_seed(D)
    n, k = heads * D, kv * D
    Q, K = torch.randn(200, n, generator=g), 2.0 + torch.randn(300, k, generator=g)
    V = (1 << 19) // D + torch.randint(-8, 9, (300, k), generator=g).float()
    dO = torch.randint(0, 3, (200, n), generator=g).float()
    a = Attention(blk.indptr, blk.indices, Q, K, V, heads, kv, D ** -0.5).backward(dO)
    dQ = B.fastgl_attn_bwd(dev_i32(blk.indptr), dev_i32(blk.indices), Q.cuda(), K.cuda(), V.cuda(), dO.cuda(), heads, kv, want=("dQ",))[0]
    u, k1 = a.u, a.k[a.v].abs()
    dp = (dO.double().reshape(200, heads, D)[u] * a.x[a.v]).sum(2)
    assert float(dp.abs().max()) < 2 ** 24 and float(dp.max()) > 2 ** 18
    rows = u[:, None].expand(-1, heads)
    high, low = (torch.zeros(200, heads, dtype=torch.float64).scatter_reduce_(0, rows, dp, f, include_self=False) for f in ("amax", "amin"))
    spread = (high - low)[:, :, None]                             # of dp in a row: what any of them less another is at most
    pk = a.to_rows(a.p[:, :, None] * k1)
    off_p = a.off_s + a.off_lse[u]                                # relative errors of the weights, and what they make of dp - delta
    weights = a.to_rows((a.p * off_p)[:, :, None] * k1) + a.to_rows(a.p * off_p)[:, :, None] * pk
    # sums of n terms of dp less another of the row's, and as many joined parts, each brought to another's reference: three roundings
    bound = a.scale * spread * (weights + 3 * U32 * (a.n + 40)[:, :, None] * pk) + 4 * U32 * a.dQ.abs()
    got = dQ.double().cpu().reshape(a.dQ.shape)
    bad = (got - a.dQ).abs() > bound
    assert not bool(bad.any()), (int(bad.sum()), (got - a.dQ).abs()[bad][:4], bound[bad][:4])
    long = a.n[:, 0] >= 4
    assert float(bound[long].median()) < 0.05 * float(a.dQ[long].abs().median())          # the check can fail


@pytest.mark.parametrize("heads,kv,D", [(1, 1, 3), (4, 2, 8), (3, 3, 20), (2, 1, 64), (2, 2, 160)])
def test_an_edge_of_no_weight_is_no_reference(heads, kv, D):
    """The first edge of a row, and one inside, have values far from the others' and weights of e^-60: they are worth nothing in dQ, nor is what is subtracted for them."""
    blk = bg.random_block(np.random.default_rng(D), 200, 300, 6.0, empty_frac=0.1, hub_rows=4, hub_deg=900)
    g = torch.Generator().manual_seed(D)
    n, k = heads * D, kv * D
    col = torch.as_tensor(blk.indices).long() % 290
    ptr = torch.as_tensor(blk.indptr).long()
    bucket = torch.zeros(blk.num_edges, dtype=torch.int32)
    for a, b in zip(ptr[:-1].tolist(), ptr[1:].tolist()):
        for e in {a, (a + b) // 2} if b - a > 3 else ():
            col[e], bucket[e] = 290 + e % 10, 1
    bias = torch.tensor([[0.0], [-60.0]]).repeat(1, heads)
    Q, K = torch.randn(200, n, generator=g) / 4, 2.0 + torch.randn(300, k, generator=g)
    V = torch.randint(-8, 9, (300, k), generator=g).float()
    V[290:] = (1 << 19) // D
    dO = torch.randint(0, 3, (200, n), generator=g).float()
    a = Attention(blk.indptr, col, Q, K, V, heads, kv, D ** -0.5, bucket, bias).backward(dO)
    dQ = B.fastgl_attn_bwd(dev_i32(blk.indptr), col.int().cuda(), Q.cuda(), K.cuda(), V.cuda(), dO.cuda(), heads, kv, bucket=bucket.cuda(), bias=bias.cuda(),
                           want=("dQ",))[0]
    u, k1 = a.u, a.k[a.v].abs()
    dp = (dO.double().reshape(200, heads, D)[u] * a.x[a.v]).sum(2)
    from_mean = (dp - a.to_rows(a.p * dp)[u]).abs()
    off_p = a.off_s + a.off_lse[u]
    widest = torch.zeros(200, heads, D, dtype=torch.float64).scatter_reduce_(0, u[:, None, None].expand(-1, heads, D), k1, "amax")
    # weights: as above, of what is left of dp.  Sums: a running mean of the first t edges is off the row's by at most B / (their weight), B = sum p |dp - delta|,
    # so that an edge's terms and what it moves the mean by are at most some 4 B of K's largest element, each rounded three times
    # The reference is a float: rounded, and from a reciprocal that is off by 2^-23, it is up to 2^-22 of itself off the mean, and so is every dp of a row that
    # has one value alone: what is left of such terms cancels but for their own rounding (seen where all that B has is e^-60 2^19 = 5e-21).
    B_ = (a.to_rows(a.p * from_mean) + 2.0 ** -22 * a.to_rows(a.p * dp).abs())[:, :, None]
    weights = a.to_rows((a.p * off_p * from_mean)[:, :, None] * k1) + a.to_rows(a.p * off_p * from_mean)[:, :, None] * widest
    bound = a.scale * (weights + 12 * U32 * (a.n + 40)[:, :, None] * B_ * widest) + 4 * U32 * a.dQ.abs()
    got = dQ.double().cpu().reshape(a.dQ.shape)
    bad = (got - a.dQ).abs() > bound
    assert not bool(bad.any()), (int(bad.sum()), (got - a.dQ).abs()[bad][:4], bound[bad][:4])
    some = (a.n[:, 0] >= 4) & (a.n[:, 0] < 100)
    assert float(bound[some].median()) < 0.05 * float(a.dQ[some].abs().median())
