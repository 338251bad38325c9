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


def test_attention_of_more_workgroups_than_a_launch_has_in_one_dimension():
    """Rows of one edge: O is the neighbour's V, dV the target's dO, bit for bit."""
    n, heads, D = (1 << 23) + 3, 5, 2
    g = torch.Generator(device="cuda").manual_seed(4)
    col = torch.randperm(n, generator=g, device="cuda", dtype=torch.int32)
    ptr = torch.arange(n + 1, device="cuda", dtype=torch.int32)
    Q, K, V, dO = (torch.randn(n, heads * D, generator=g, device="cuda").bfloat16() for _ in range(4))
    bucket = torch.arange(n, device="cuda", dtype=torch.int32) % 3
    how = dict(heads=heads, bucket=bucket, bias=torch.zeros(3, heads, device="cuda"))
    O, lse = B.fastgl_attn_fwd(ptr, col, Q, K, V, **how)
    assert torch.equal(O, V[col.long()]) and bool(torch.isfinite(lse).all())
    dQ, dK, dV, dbias = B.fastgl_attn_bwd(ptr, col, Q, K, V, dO, **how)
    assert torch.equal(dV[col.long()], dO) and float(dQ.abs().max()) < 2.0 ** -14


def test_a_bias_of_very_many_buckets_and_heads():
    """A row of one edge (its gradient is 0) and one of two, whose gradients are in the table's last rows."""
    heads, buckets = 4096, 65536
    g = torch.Generator(device="cuda").manual_seed(5)
    ptr = torch.tensor([0, 1, 3], device="cuda", dtype=torch.int32)
    col = torch.tensor([0, 1, 2], device="cuda", dtype=torch.int32)
    Q, K, V, dO = (torch.randn(r, heads, generator=g, device="cuda") for r in (2, 3, 3, 2))
    bucket = torch.tensor([7, buckets - 1, buckets - 2], device="cuda", dtype=torch.int32)
    bias = torch.zeros(buckets, heads, device="cuda")
    dbias = B.fastgl_attn_bwd(ptr, col, Q, K, V, dO, heads=heads, bucket=bucket, bias=bias)[3]
    s = (Q[1] * K[1:]).double()
    p = torch.softmax(s, 0)
    dp = (dO[1] * V[1:]).double()
    ds = p * (dp - (p * dp).sum(0))
    # scores below 32, |dp| below 32: a weight is off by 2^-23 (2 + |s|) and dp's difference by 2^-22 of it
    torch.testing.assert_close(dbias[-2:].flip(0).double(), ds, rtol=0, atol=2.0 ** -23 * 40 * 64)
    assert not bool(dbias[:-2].any())


def test_the_loss_of_half_a_billion_rows():
    M, N = (1 << 29) + 5, 2
    g = torch.Generator(device="cuda").manual_seed(6)
    H = torch.randn(M, 1, generator=g, device="cuda", dtype=torch.bfloat16)
    W, b = torch.randn(1, N, generator=g, device="cuda").bfloat16(), torch.zeros(N, device="cuda")
    label = torch.randint(-1, N, (M,), generator=g, device="cuda")
    loss, lse = B.fastgl_loss_fwd(H, W, b, label)
    for at in (0, M // 2, M - 100_000):
        part = slice(at, at + 100_000)
        ref = Loss(H[part], W, b, label[part])
        for got, name in ((loss[part], "loss"), (lse[part], "lse")):
            want, off = getattr(ref, name), getattr(ref, "off_" + name)
            assert not bool(((got.double() - want).abs() > off + 2.0 ** -24 * (want.abs() + off)).any()), (name, at)


def test_row_gradients_of_four_billion_elements():
    """dH of 2^32 elements from two pieces of the classes, whose sums are joined."""
    M, K, N = (1 << 25) + 3, 128, 300
    g = torch.Generator(device="cuda").manual_seed(7)
    H = torch.randn(M, K, generator=g, device="cuda", dtype=torch.bfloat16)
    W, b = (torch.randn(K, N, generator=g, device="cuda") / 8).bfloat16(), torch.zeros(N, device="cuda")
    label, dloss = torch.randint(-1, N, (M,), generator=g, device="cuda"), torch.randn(M, generator=g, device="cuda")
    _, lse = B.fastgl_loss_fwd(H, W, b, label)
    dH = B.fastgl_loss_bwd(H, W, b, label, lse, dloss, want=("dH",))[0]
    for at in (0, M // 2, M - 5000):
        part = slice(at, at + 5000)
        ref = Loss(H[part], W, b, label[part]).backward(dloss[part])
        off = ref.off_dH
        assert not bool(((dH[part].double() - ref.dH).abs() > off + 2.0 ** -8 * (ref.dH.abs() + off)).any()), at
