"""The plain form of the gated update against differences, the piece products in numpy, and the entry points' refusals."""
import ctypes

import numpy as np
import pytest
import torch

import gated_ref as ref
from paper_2409_14939_amd import binding as B


@pytest.mark.parametrize("name", ref.ACTS)
def test_gradient_against_differences(name):
    gen = torch.Generator().manual_seed(1)
    x, wg, wu = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((5, 4), (4, 6), (4, 6)))
    bg, bu = (torch.randn(6, generator=gen, dtype=torch.float64) for _ in range(2))
    dp = torch.randn(5, 6, generator=gen, dtype=torch.float64)
    _, g, u = ref.forward(x, wg, wu, bg, bu, name)
    grads = ref.backward(x, wg, wu, g, u, dp, name)[:5]

    def loss():
        return (ref.forward(x, wg, wu, bg, bu, name)[0] * dp).sum().item()
    for v, grad in zip((x, wg, wu, bg, bu), grads):
        flat = v.view(-1)
        for i in range(flat.numel()):
            keep, step = flat[i].item(), 1e-6
            flat[i] = keep + step
            up = loss()
            flat[i] = keep - step
            down = loss()
            flat[i] = keep
            assert abs((up - down) / (2 * step) - grad.reshape(-1)[i].item()) < 1e-6


def test_series_of_the_normal_distribution():
    """The five-term series the kernels use is within 1.5e-7 of erfc, in 64 bits."""
    x = torch.linspace(0, 8, 20_001, dtype=torch.float64)
    t = 1 / (1 + 0.3275911 * x)
    a = (0.254829592, -0.284496736, 1.421413741, -1.453152027, 1.061405429)
    poly = sum(c * t ** (i + 1) for i, c in enumerate(a))
    assert (poly * torch.exp(-x * x) - torch.special.erfc(x)).abs().max() < 1.5e-7


def test_six_of_nine_piece_products_leave_a_unit_of_float32():
    rng = np.random.default_rng(0)
    a, b = (rng.standard_normal(20_000).astype(np.float32) for _ in range(2))

    def cut(x):
        out = []
        for _ in range(3):
            p = torch.from_numpy(x).bfloat16().float().numpy()
            out.append(p.astype(np.float64))
            x = x - p
        assert not x.any()                                      # the three pieces are the element
        return out
    pa, pb = cut(a), cut(b)
    got = sum(pa[i] * pb[j] for i, j in ((0, 2), (2, 0), (1, 1), (0, 1), (1, 0), (0, 0)))
    want = a.astype(np.float64) * b.astype(np.float64)
    assert np.max(np.abs(got - want) / np.abs(want)) <= 2.0 ** -23


FAKE, ODD, TWO = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001), ctypes.c_void_p(0x1002)
INVALID, UNSUPPORTED, WORKSPACE = B.FASTGL_ERR_INVALID_ARG, B.FASTGL_ERR_UNSUPPORTED, B.FASTGL_ERR_WORKSPACE


def fwd(dt=1, X=FAKE, Wg=FAKE, Wu=FAKE, bg=None, bu=None, M=64, K=8, N=8, act=0, P=FAKE, G=None, U=None, ws=FAKE, wsb=1 << 40):
    return B.lib().fastgl_gated_fwd(dt, X, Wg, Wu, bg, bu, M, K, N, act, P, G, U, ws, wsb, None)


def bwd(dt=1, X=FAKE, Wg=FAKE, Wu=FAKE, G=FAKE, U=FAKE, dP=FAKE, M=64, K=8, N=8, act=0, dX=FAKE, dWg=FAKE, dWu=FAKE, dbg=None, dbu=None,
        ws=FAKE, wsb=1 << 40):
    return B.lib().fastgl_gated_bwd(dt, X, Wg, Wu, G, U, dP, M, K, N, act, dX, dWg, dWu, dbg, dbu, ws, wsb, None)


@pytest.mark.parametrize("call,kw,status,text", [
    *[(f, kw, s, t) for f in (fwd, bwd) for kw, s, t in (
        (dict(dt=2), INVALID, "dtype"), (dict(act=4), INVALID, "activation"), (dict(act=-1), INVALID, "activation"),
        (dict(M=-1), INVALID, "negative"), (dict(K=-1), INVALID, "negative"), (dict(N=-1), INVALID, "negative"),
        (dict(M=2 ** 31 - 1), UNSUPPORTED, "2^31"), (dict(K=2 ** 20 + 1), UNSUPPORTED, "2^20"), (dict(N=2 ** 20 + 1), UNSUPPORTED, "2^20"),
        (dict(X=ODD), INVALID, "aligned"), (dict(dt=0, Wg=TWO), INVALID, "aligned"), (dict(Wu=ODD), INVALID, "aligned"))],
    *[(fwd, {k: None}, INVALID, "NULL") for k in ("X", "Wg", "Wu", "P")],
    *[(fwd, {k: TWO}, INVALID, "aligned") for k in ("bg", "bu")], (fwd, dict(P=ODD), INVALID, "aligned"), (fwd, dict(G=ODD), INVALID, "aligned"),
    (fwd, dict(dt=0, ws=None), INVALID, "workspace"), (fwd, dict(dt=0, ws=ctypes.c_void_p(0x1010)), INVALID, "workspace"),
    (fwd, dict(dt=0, wsb=64), WORKSPACE, "too small"), (fwd, dict(K=9, wsb=64), WORKSPACE, "too small"), (fwd, dict(N=9, wsb=64), WORKSPACE, "too small"),
    (fwd, dict(X=TWO, wsb=64), WORKSPACE, "too small"),
    *[(bwd, {k: None}, INVALID, "NULL") for k in ("G", "U", "dP")], (bwd, dict(X=None), INVALID, "need X"), (bwd, dict(Wg=None), INVALID, "needs Wg"),
    (bwd, dict(dbg=TWO), INVALID, "aligned"), (bwd, dict(ws=None), INVALID, "workspace"), (bwd, dict(wsb=64), WORKSPACE, "too small"),
])
def test_bad_arguments_are_refused_before_launch(call, kw, status, text):
    assert call(**kw) == status
    assert text in B.fastgl_last_error()


def test_calls_with_nothing_to_do():
    assert fwd(M=0, X=None, P=None) == B.FASTGL_OK and fwd(N=0, Wg=None, Wu=None, P=None) == B.FASTGL_OK
    assert bwd(dX=None, dWg=None, dWu=None, G=None, U=None, dP=None, X=None) == B.FASTGL_OK


def test_workspace_sizes():
    f, b = B.fastgl_gated_fwd_workspace_bytes, B.fastgl_gated_bwd_workspace_bytes
    assert f("bf16", 1000, 64, 64, True) == 0 and f("bf16", 1000, 64, 64, False) > 0
    assert f("bf16", 1000, 65, 64, True) >= 2 * 1000 * 72 and f("bf16", 1000, 64, 65, True) >= 2 * 2 * 64 * 72
    assert f("f32", 1000, 64, 64, True) >= 6 * (1000 * 64 + 2 * 64 * 64) and f("f32", 1, 64, 64) == 0
    assert b("bf16", 1000, 64, 64, True) >= 2 * 2 * 1000 * 64 and b("f32", 1000, 64, 64, True) >= 3 * b("bf16", 1000, 64, 64, True) // 2
    assert f("bf16", -1, 8, 8) == 0 and b("bf16", 8, -1, 8) == 0 and b("bf16", 8, 8, 2 ** 21) == 0
    for M, K, N in ((16_384, 1024, 4096), (1, 2 ** 20, 2 ** 20), (300_000, 64, 64)):
        assert b("bf16", M, K, N) < 40 * (M * (K + 2 * N) + 4 * K * N) + (1 << 26)


def test_fine_calls_are_checked_alike():
    def fine(dt=1, M=64, K=8, N=8, act=0, G=FAKE, X=FAKE, ws=FAKE, wsb=1 << 40):
        return B.lib().fastgl_gated_bwd_fine(dt, X, FAKE, FAKE, G, FAKE, FAKE, M, K, N, act, FAKE, FAKE, FAKE, None, None, ws, wsb, None)
    for kw, status in ((dict(dt=2), INVALID), (dict(act=4), INVALID), (dict(M=-1), INVALID), (dict(K=2 ** 20 + 1), UNSUPPORTED), (dict(G=None), INVALID),
                       (dict(X=ODD), INVALID), (dict(ws=None), INVALID), (dict(wsb=64), WORKSPACE)):
        assert fine(**kw) == status
    size = B.fastgl_gated_bwd_workspace_bytes
    for M, K, N in ((1, 8, 16), (300, 33, 32), (5000, 256, 683)):
        assert size("bf16", M, K, N, fine=True) >= 2 * 2 * 2 * M * N                           # two pieces of both
        assert size("f32", M, K, N, fine=True) == size("f32", M, K, N)
    assert fine(M=300, K=33, N=32, wsb=size("bf16", 300, 33, 32)) == WORKSPACE
