"""Attention and the loss between bands of a sentinel: results and workspaces of the stated size and no byte more; two streams at once."""
import numpy as np
import pytest
import torch

import blockgen as bg
from gpu_util import dev_i32
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BAND, SENTINEL = 4096, 0xA5


class Bands:
    """Arrays in the middle of larger ones."""

    def __init__(self):
        self.all = []

    def make(self, shape, dtype, shift=0):
        n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        whole = torch.full((n + 2 * BAND,), SENTINEL, dtype=torch.uint8, device="cuda")
        self.all.append((whole, BAND + shift, n))
        return whole[BAND + shift:BAND + shift + n].view(dtype).reshape(shape)

    def check(self):
        for i, (whole, at, n) in enumerate(self.all):
            assert bool((whole[:at] == SENTINEL).all()) and bool((whole[at + n:] == SENTINEL).all()), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,D,buckets", [(1, 1, 1, 3), (4, 2, 16, None), (4, 2, 16, 0), (3, 1, 47, 70), (2, 2, 200, 2)])
def test_attention_writes_what_is_its_own(heads, kv, D, buckets, dtype):
    blk = bg.random_block(np.random.default_rng(heads), 301, 413, 4.0, empty_frac=0.2, hub_rows=3, hub_deg=700)
    t = DTYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(1)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").to(t)
    n, k, E = heads * D, kv * D, blk.num_edges
    block = dev_i32(blk.indptr), dev_i32(blk.indices)
    Q, K, V, dO = make(301, n), make(413, k), make(413, k), make(301, n)
    how = dict(heads=heads, kv_heads=kv)
    if buckets is not None:
        how["bucket"] = torch.randint(-1, buckets + 1, (E,), generator=g, device="cuda", dtype=torch.int32)
    if buckets:
        how["bias"] = torch.randn(buckets, heads, generator=g, device="cuda")
    need = [B.fastgl_attn_workspace_bytes(301, 413, E, heads, D, dtype, kv_heads=kv, num_buckets=buckets or 0, backward=b, bucket=buckets == 0) for b in (False, True)]
    bands = Bands()
    el = 2 if dtype == "bf16" else 4
    into = [bands.make(s, x, el if x == t else 0) for s, x in (((301, n), t), ((301, heads), torch.float32), ((301, n), t), ((413, k), t), ((413, k), t))]
    dbias = bands.make((buckets, heads), torch.float32) if buckets else None
    ws = [bands.make((b,), torch.uint8) for b in need]
    plain = [*B.fastgl_attn_fwd(*block, Q, K, V, **how), *B.fastgl_attn_bwd(*block, Q, K, V, dO, **how)]
    got = [*B.fastgl_attn_fwd(*block, Q, K, V, **how, O=into[0], lse=into[1], workspace=ws[0]),
           *B.fastgl_attn_bwd(*block, Q, K, V, dO, **how, dQ=into[2], dK=into[3], dV=into[4], dbias=dbias, workspace=ws[1])]
    assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(plain, got))
    bands.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, 5, 3), (33, 40, 65), (300, 72, 1000), (1000, 300, 77), (2000, 513, 1031), (8200, 512, 130)])
def test_the_loss_writes_what_is_its_own(M, K, N, dtype):
    t = DTYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(1)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")
    H, W, b, dloss = make(M, K).to(t), (make(K, N) / K ** 0.5).to(t), make(N), make(M)
    label = torch.randint(-1, N, (M,), generator=g, device="cuda")
    bands = Bands()
    el = 2 if dtype == "bf16" else 4
    f32 = torch.float32
    loss, lse, dH, dW, db = (bands.make(s, x, el if x == t else 4) for s, x in (((M,), f32), ((M,), f32), ((M, K), t), ((K, N), t), ((N,), f32)))
    aligned = H.data_ptr() % 16 == 0 and W.data_ptr() % 16 == 0
    ws = [bands.make((f(dtype, M, K, N, aligned),), torch.uint8) for f in (B.fastgl_loss_fwd_workspace_bytes, B.fastgl_loss_bwd_workspace_bytes)]
    first = B.fastgl_loss_fwd(H, W, b, label)
    plain = [*first, *B.fastgl_loss_bwd(H, W, b, label, first[1], dloss)]
    got = [*B.fastgl_loss_fwd(H, W, b, label, loss=loss, lse=lse, workspace=ws[0]),
           *B.fastgl_loss_bwd(H, W, b, label, lse, dloss, dH=dH, dW=dW, db=db, workspace=ws[1])]
    assert all(torch.equal(a, x) for a, x in zip(plain, got))
    bands.check()


def test_two_streams_at_once():
    """Calls that share nothing but their inputs."""
    blk = bg.random_block(np.random.default_rng(2), 4000, 6000, 9.0, hub_rows=4, hub_deg=2000)
    g = torch.Generator(device="cuda").manual_seed(1)
    block = dev_i32(blk.indptr), dev_i32(blk.indices)
    Q, K, V, dO = (torch.randn(r, 64, generator=g, device="cuda") for r in (4000, 6000, 6000, 4000))
    how = dict(heads=4, bucket=torch.randint(-1, 5, (blk.num_edges,), generator=g, device="cuda", dtype=torch.int32), bias=torch.randn(5, 4, generator=g, device="cuda"))
    W, label, dloss = torch.randn(64, 300, generator=g, device="cuda"), torch.randint(-1, 300, (4000,), generator=g, device="cuda"), torch.rand(4000, generator=g, device="cuda")

    def step():
        O, lse = B.fastgl_attn_fwd(*block, Q, K, V, **how)
        loss, z = B.fastgl_loss_fwd(O, W, None, label)
        return [O, lse, loss, z, *B.fastgl_loss_bwd(O, W, None, label, z, dloss), *B.fastgl_attn_bwd(*block, Q, K, V, dO, **how)]
    want = step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                results.append(step())
    torch.cuda.synchronize()
    for got in results:
        assert all(torch.equal(a, b) for a, b in zip(want, got))
