"""The operators of examples/residual_block.py together: gradients of the whole chain against differences, both types, and the
rows of the 8-bit table."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import blockgen as bg
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("residual_block", os.path.join(ROOT, "examples", "residual_block.py"))
ex = importlib.util.module_from_spec(spec)
spec.loader.exec_module(ex)
WIDTH, HIDDEN, CLASSES, P = 44, 91, 7, 0.3


def setting(dtype):
    blk = bg.make_config(1).blocks[0]
    ip, ix = torch.from_numpy(blk.indptr).cuda(), torch.from_numpy(blk.indices).cuda()
    g = torch.Generator().manual_seed(1)
    X = torch.randn(blk.num_src, WIDTH, generator=g).to(dtype).cuda()
    dlogits = torch.randn(blk.num_dst, CLASSES, generator=g).to(dtype).cuda()
    return (ip, ix, B.fastgl_block_plan_create(ip, ix, blk.num_src)), X, dlogits


def test_gradients_of_the_chain_against_differences():
    block, X, dlogits = setting(torch.float32)
    q, states = ex.make_params(WIDTH, HIDDEN, CLASSES, torch.float32), ex.rng_states(7, 2 ** 40)
    _, kept = ex.forward(q, block, X, states, P)
    grads, dX = ex.backward(q, block, X, kept, dlogits, states, P)

    def loss(q, X):
        return (ex.forward(q, block, X, states, P)[0].double() * dlogits.double()).sum().item()
    gen = torch.Generator().manual_seed(5)
    for name in [*grads, "X"]:
        v, g = (X, dX) if name == "X" else (q[name], grads[name])
        # along the gradient itself and a random direction: the change is far above the logits' float32 noise
        way = g.double() / g.double().norm() + 0.5 * torch.randn(v.shape, generator=gen, dtype=torch.float64).cuda() / v.numel() ** 0.5
        step = 1e-2 * max(v.double().norm().item(), 1.0) / way.norm().item() / 10
        up, down = (v.double() + step * way).float(), (v.double() - step * way).float()
        along = ((up.double() - down.double()) * g.double()).sum().item()
        if name == "X":
            change = loss(q, up) - loss(q, down)
        else:
            change = loss({**q, name: up}, X) - loss({**q, name: down}, X)
        # third-order term of a central difference over a thousandth of the parameter's size, and float32 noise
        assert abs(change - along) <= 1e-2 * abs(along) + 1e-3, (name, change, along)


def test_both_types_agree():
    out = []
    for dtype in (torch.float32, torch.bfloat16):
        block, X, dlogits = setting(dtype)
        q, states = ex.make_params(WIDTH, HIDDEN, CLASSES, dtype), ex.rng_states(7, 3)
        logits, kept = ex.forward(q, block, X, states, P)
        grads, dX = ex.backward(q, block, X, kept, dlogits, states, P)
        out.append([logits, dX, *grads.values()])
    for a, b in zip(*out):
        # inputs, weights and some ten results on the way are rounded to 8 bits (2^-8 each, independent)
        assert ((a.double() - b.double()).norm() / a.double().norm()).item() < 12 * 2.0 ** -8


def test_rows_of_the_table():
    block, X, _ = setting(torch.bfloat16)
    q, states = ex.make_params(WIDTH, HIDDEN, CLASSES, torch.bfloat16), ex.rng_states(1, 1)
    _, kept = ex.forward(q, block, X, states, 0.0)
    Q, scale = ex.table_of(q, kept)
    ids = torch.arange(Q.shape[0] - 1, -1, -3, device="cuda")
    for dtype, half in (("f32", 0.0), ("bf16", 2.0 ** -8)):
        rows = B.fastgl_gather_rows_e4m3(Q, scale, ids, dtype).double()
        y = kept["z"].double()
        y = (y / torch.sqrt(y.square().mean(1, keepdim=True) + ex.EPS))[ids]
        bound = y.abs() * (2.0 ** -4 * 1.001 + half) + scale.double()[ids][:, None] * 2.0 ** -10 * 1.01
        assert bool(((rows - y).abs() <= bound).all())
    assert np.isfinite(rows.cpu().numpy()).all()


def test_a_mini_batch_of_reused_rows_and_rows_of_an_8_bit_table():
    """Match, the gather of what has to be loaded, assembly: the same calls as with a float32 table, and the same rows as a gather of all."""
    g = torch.Generator().manual_seed(3)
    rows, F = 5000, 100
    table = torch.randn(rows, F, generator=g).cuda()
    Q, scale, _, _ = B.fastgl_norm_fwd_e4m3(table, torch.ones(F).cuda(), ex.EPS, want_rstd=False)
    first, second = (torch.randperm(rows, generator=g)[:n].cuda() for n in (1500, 1777))
    for dtype in ("f32", "bf16"):
        X = B.fastgl_gather_rows_e4m3(Q, scale, first, dtype)
        src_row, _, load_gid, result = B.fastgl_match(first, second)
        n_load, violations = result.tolist()
        assert violations == 0 and 0 < n_load < second.numel()
        load = B.fastgl_gather_rows_e4m3(Q, scale, load_gid[:n_load], dtype)
        assert torch.equal(B.fastgl_assemble_rows(X, load, src_row, n_load), B.fastgl_gather_rows_e4m3(Q, scale, second, dtype))
