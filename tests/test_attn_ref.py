"""Attention over a block's edges on the CPU: its gradients against differences, and what the entry points refuse."""
import ctypes

import numpy as np
import pytest
import torch

import blockgen as bg
from attn_ref import Attention
from paper_2409_14939_amd import binding as B


@pytest.mark.parametrize("shared", [1, 3])
def test_gradients_against_differences(shared):
    g = torch.Generator().manual_seed(1)
    blk = bg.random_block(np.random.default_rng(2), 7, 11, 3.0)
    kv, D = 2, 4
    heads = kv * shared
    make = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    Q, K, V, dO, bias = make(7, heads * D), make(11, kv * D), make(11, kv * D), make(7, heads * D), make(3, heads)
    bucket = torch.randint(-1, 3, (blk.num_edges,), generator=g)

    def loss():
        a = Attention(blk.indptr, blk.indices, Q, K, V, heads, kv, 0.7, bucket, bias)
        return (a.O.reshape(7, -1) * dO).sum().item()
    a = Attention(blk.indptr, blk.indices, Q, K, V, heads, kv, 0.7, bucket, bias).backward(dO)
    for x, grad in ((Q, a.dQ), (K, a.dK), (V, a.dV), (bias, a.dbias)):
        flat, want = x.view(-1), grad.reshape(-1)
        for i in range(flat.numel()):
            keep = flat[i].item()
            flat[i] = keep + 1e-6
            up = loss()
            flat[i] = keep - 1e-6
            down = loss()
            flat[i] = keep
            assert abs((up - down) / 2e-6 - want[i].item()) < 1e-7


def test_softmax_of_a_row_by_hand():
    Q, K, V = torch.tensor([[1.0, 0.0]]), torch.tensor([[0.0, 5.0], [np.log(3.0), 1.0]]).float(), torch.tensor([[4.0, 0.0], [0.0, 8.0]])
    a = Attention([0, 2], [0, 1], Q, K, V, 1, 1, 1.0)
    assert torch.allclose(a.O.reshape(-1), torch.tensor([1.0, 6.0], dtype=torch.float64), atol=1e-6)
    assert abs(a.lse.item() - np.log(4.0)) < 1e-6


FAKE, ODD, TWO = 0x1000, 0x1001, 0x1002
INVALID, UNSUPPORTED, WORKSPACE = B.FASTGL_ERR_INVALID_ARG, B.FASTGL_ERR_UNSUPPORTED, B.FASTGL_ERR_WORKSPACE


def desc(**kw):
    d = dict(indptr=FAKE, indices=FAKE, num_dst=4, num_src=6, num_edges=9, bucket=None, bias=None, num_buckets=0, heads=4, kv_heads=2, width=8,
             scale=1.0, dtype=1, Q=FAKE, K=FAKE, V=FAKE, ldq=32, ldk=16, ldv=16)
    return B.AttnDesc(**{**d, **{k: v for k, v in kw.items() if k in d}}), {k: v for k, v in kw.items() if k not in d}


def fwd(**kw):
    d, more = desc(**kw)
    a = {**dict(O=FAKE, ldo=32, lse=FAKE, plan=None, ws=FAKE, wsb=1 << 40), **more}
    return B.lib().fastgl_attn_fwd(ctypes.byref(d), a["O"], a["ldo"], a["lse"], a["plan"], a["ws"], a["wsb"], None)


def bwd(**kw):
    d, more = desc(**kw)
    a = {**dict(dO=FAKE, lddo=32, dQ=FAKE, lddq=32, dK=FAKE, lddk=16, dV=FAKE, lddv=16, dbias=None, plan=None, ws=FAKE, wsb=1 << 40), **more}
    return B.lib().fastgl_attn_bwd(ctypes.byref(d), *(a[k] for k in ("dO", "lddo", "dQ", "lddq", "dK", "lddk", "dV", "lddv", "dbias", "plan",
                                                                     "ws", "wsb")), None)


BOTH = [
    (dict(num_dst=-1), INVALID, "negative"), (dict(num_src=-1), INVALID, "negative"), (dict(num_edges=-1), INVALID, "negative"),
    (dict(num_buckets=-1), INVALID, "negative"), (dict(num_dst=2 ** 31 - 1), UNSUPPORTED, "2^31"), (dict(num_edges=2 ** 31 - 1), UNSUPPORTED, "2^31"),
    (dict(num_src=0), INVALID, "at least one"), (dict(dtype=2), INVALID, "dtype"), (dict(heads=0), INVALID, "heads"), (dict(kv_heads=0), INVALID, "heads"),
    (dict(kv_heads=3), INVALID, "multiple"), (dict(width=0), INVALID, "width"), (dict(width=257, ldq=2000, ldk=2000, ldv=2000), UNSUPPORTED, "256"),
    (dict(heads=4098, kv_heads=4098, width=1, ldq=9999, ldk=9999, ldv=9999), UNSUPPORTED, "4096"),
    (dict(heads=512, kv_heads=2, width=256, ldq=1 << 20, ldk=512, ldv=512), UNSUPPORTED, "65536"),
    (dict(bias=FAKE, num_buckets=3), INVALID, "buckets"), (dict(bias=FAKE, bucket=FAKE), INVALID, "buckets"),
    (dict(bias=FAKE, bucket=FAKE, num_buckets=65_537), UNSUPPORTED, "65536"), (dict(indptr=None), INVALID, "NULL"), (dict(indices=None), INVALID, "NULL"),
    (dict(Q=None), INVALID, "NULL"), (dict(K=None), INVALID, "NULL"), (dict(V=None), INVALID, "NULL"), (dict(ldq=31), INVALID, "ldq"), (dict(ldk=15), INVALID, "ldk"),
    (dict(ldv=15), INVALID, "ldv"), (dict(Q=ODD), INVALID, "aligned"), (dict(dtype=0, K=TWO), INVALID, "aligned"), (dict(V=ODD), INVALID, "aligned"),
    (dict(indptr=TWO), INVALID, "aligned"), (dict(indices=TWO), INVALID, "aligned"), (dict(bucket=TWO), INVALID, "aligned"),
    (dict(bucket=FAKE, bias=TWO, num_buckets=3), INVALID, "aligned"), (dict(num_edges=1000, ws=None), INVALID, "workspace"),
    (dict(num_edges=1000, ws=0x1010), INVALID, "workspace"), (dict(num_edges=1000, wsb=64), WORKSPACE, "too small")]


@pytest.mark.parametrize("call,kw,status,text", [
    *[(f, *c) for f in (fwd, bwd) for c in BOTH],
    (fwd, dict(O=None), INVALID, "NULL"), (fwd, dict(O=ODD), INVALID, "misaligned"), (fwd, dict(ldo=31), INVALID, "ldo"), (fwd, dict(lse=TWO), INVALID, "misaligned"),
    (bwd, dict(dO=None), INVALID, "NULL"), (bwd, dict(dbias=FAKE), INVALID, "dbias"),
    *[(bwd, {k: 15}, INVALID, "row's length") for k in ("lddo", "lddq", "lddk", "lddv")],
    *[(bwd, {k: ODD}, INVALID, "aligned") for k in ("dO", "dQ", "dK", "dV")],
    (bwd, dict(bucket=FAKE, bias=FAKE, num_buckets=3, dbias=TWO), INVALID, "aligned"), (bwd, dict(ws=None), INVALID, "workspace")])
def test_bad_arguments_are_refused_before_launch(call, kw, status, text):
    assert call(**kw) == status
    assert text in B.fastgl_last_error()


def test_calls_with_nothing_to_do():
    assert fwd(num_dst=0, num_edges=0, Q=None, O=None) == B.FASTGL_OK
    assert bwd(dQ=None, dK=None, dV=None, dO=None) == B.FASTGL_OK
    assert B.lib().fastgl_attn_fwd(None, FAKE, 8, None, None, None, 0, None) == INVALID


def test_workspace_sizes():
    size = B.fastgl_attn_workspace_bytes
    assert size(1, 16, 15, 4, 64, "bf16") == 0                       # no row can be long
    assert size(1000, 1000, 10_000, 4, 64, "bf16") >= (10_000 // 128) * 4 * 64 * 4
    assert size(1000, 1000, 10_000, 4, 64, "bf16", backward=True) > 2 * (10_000 // 128) * 4 * 64 * 4 + 1000 * 4 * 4
    more = size(1000, 1000, 10_000, 4, 64, "f32", num_buckets=100, backward=True)
    assert more >= size(1000, 1000, 10_000, 4, 64, "f32", backward=True) + 10_000 * 4 * 4 + 100 * 4 * 4
    assert size(10, 10, 10, 4, 300, "f32") == 0 and size(10, 10, 10, 4, 8, "f32", kv_heads=3) == 0
    assert size(2 ** 20, 2 ** 20, 2 ** 24, 64, 4, "f32", num_buckets=65_536, backward=True) < 2 ** 24 * 64 * 4 + 2 ** 20 * 64 * 16 + (5 << 28)
