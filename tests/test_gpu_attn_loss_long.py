"""Attention over arrays whose offsets pass 32 bits, and the loss of very many rows and classes."""
import numpy as np
import pytest
import torch

from gpu_util import dev_i32
from loss_ref import HALF, Loss
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv,D", [(4, 2, 64), (3, 3, 47), (2, 1, 5)])
def test_rows_beyond_four_gigabytes(heads, kv, D):
    """Neighbours at both ends of an array of more than 2^32 bytes: the same bits as from rows that lie close together."""
    nd, wide, rows = 300, 8192, (1 << 32) // (8192 * 2) + 700
    n, k = heads * D, kv * D
    far = torch.empty(rows, wide, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    ends = torch.cat((torch.arange(500), torch.arange(rows - 500, rows))).cuda()
    far[ends] = torch.randn(1000, wide, generator=g, device="cuda").bfloat16()
    degree = np.array([(7 * i) % 13 if i % 50 else 400 for i in range(nd)])
    ip = np.concatenate([[0], np.cumsum(degree)]).astype(np.int32)
    near_ix = np.random.default_rng(1).integers(0, 1000, ip[-1]).astype(np.int32)
    far_ix = ends.cpu().numpy()[near_ix].astype(np.int32)
    Q, dO = (torch.randn(nd, n, generator=g, device="cuda").bfloat16() for _ in range(2))
    bucket = torch.randint(-1, 4, (int(ip[-1]),), generator=g, device="cuda", dtype=torch.int32)
    bias = torch.randn(4, heads, generator=g, device="cuda")
    results = []
    for table, ix in ((far, far_ix), (far[ends].contiguous(), near_ix)):
        K, V = table[:, wide - 2 * k:wide - k], table[:, wide - k:]
        block = dev_i32(ip), dev_i32(ix)
        plan = B.fastgl_block_plan_create(*block, table.shape[0], B.PLAN_ALL | B.PLAN_PERM)
        how = dict(heads=heads, kv_heads=kv, bucket=bucket, bias=bias, plan=plan)
        O, lse = B.fastgl_attn_fwd(*block, Q, K, V, **how)
        dkv = torch.zeros_like(table)
        dQ, dK, dV, dbias = B.fastgl_attn_bwd(*block, Q, K, V, dO, **how, dK=dkv[:, :k], dV=dkv[:, wide - k:])
        pick = ends if table is far else torch.arange(1000, device="cuda")
        results.append((O, lse, dQ, dK[pick].clone(), dV[pick].clone(), dbias))
        if table is far:
            others = torch.ones(rows, dtype=torch.bool, device="cuda")
            others[ends] = False
            assert not bool(dkv[others][:, :k].any()) and not bool(dkv[others][:, wide - k:].any())
        assert not bool(dkv[:, k:wide - k].any())
    for i, (a, b) in enumerate(zip(*results)):
        assert bool(torch.isfinite(a).all()) or i == 1
        if i in (0, 1, 2):
            assert torch.equal(a, b), i
        else:       # sums over a source's edges, which other numbers of sources bring into another order: 2^-8 of a bf16 result
            torch.testing.assert_close(a.double(), b.double(), rtol=2.0 ** -7, atol=1e-4 * b.double().abs().max().item())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,K,N", [((1 << 21) + 300, 9, 12), ((1 << 21) + 1, 64, 40), (5, 6, 1 << 21), (300, 17, (1 << 21) - 3), (70_000, 40, 700)])
def test_many_rows_and_many_classes(M, K, N, dtype):
    g = torch.Generator(device="cuda").manual_seed(2)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")
    H, W, b = make(M, K).to(dtype), (make(K, N) / K ** 0.5).to(dtype), make(N)
    label, dloss = torch.randint(-1, N, (M,), generator=g, device="cuda"), make(M) / M
    loss, lse = B.fastgl_loss_fwd(H, W, b, label)
    grads = B.fastgl_loss_bwd(H, W, b, label, lse, dloss)
    ref = Loss(H, W, b, label).backward(dloss)
    for got, name, t in zip((loss, lse, *grads), ("loss", "lse", "dH", "dW", "db"), (torch.float32, torch.float32, dtype, dtype, torch.float32)):
        want, off = getattr(ref, name), getattr(ref, "off_" + name)
        bad = (got.double() - want).abs() > off + HALF[t] * (want.abs() + off)
        assert not bool(bad.any()), (name, int(bad.sum()))
