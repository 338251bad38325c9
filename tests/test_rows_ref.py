"""The plain forms of norm and dropout against what is known of them, and the refusals of their entry points (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import rows_ref as ref
from paper_2409_14939_amd import binding as B


@pytest.mark.parametrize("counter,key,words", [     # the generator's published known answers
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_gives_its_known_answers(counter, key, words):
    assert tuple(int(v) for v in ref.philox(*(np.uint64(c) for c in counter), *key)) == words


def test_kept_share_and_its_independence_of_the_shape():
    k = ref.keep(400, 1000, 0.3, (7, 9))
    assert abs(k.double().mean().item() - 0.7) < 5 * (0.21 / 400_000) ** 0.5
    assert torch.equal(k[:17, :333], ref.keep(17, 333, 0.3, (7, 9)))
    assert not torch.equal(k, ref.keep(400, 1000, 0.3, (7, 10))) and not torch.equal(k, ref.keep(400, 1000, 0.3, (8, 9)))
    assert ref.keep(3, 9, 0.0, (1, 1)).all() and not ref.keep(3, 9, 1.0, (1, 1)).any()


def test_gradient_against_differences():
    g = torch.Generator().manual_seed(3)
    x, r, dy, ds = (torch.randn(4, 13, generator=g, dtype=torch.float64) for _ in range(4))
    w = torch.randn(13, generator=g, dtype=torch.float64)
    state, p, eps = (5, 6), 0.3, 1e-2

    def loss(x, r, w):
        y, h, _ = ref.norm(x, w, eps, r, p, state)
        return ((y * dy).sum() + (h * ds).sum()).item()
    _, h, rstd = ref.norm(x, w, eps, r, p, state)
    got = ref.norm_grad(h, w, rstd, dy, ds, p, state)
    for k, (v, grad) in enumerate(zip((x, r, w), got)):
        flat = v.reshape(-1)
        for i in range(flat.numel()):
            keep, step = flat[i].item(), 1e-5
            flat[i] = keep + step
            up = loss(x, r, w)
            flat[i] = keep - step
            down = loss(x, r, w)
            flat[i] = keep
            assert abs((up - down) / (2 * step) - grad.reshape(-1)[i].item()) < 1e-8, (k, i)


FAKE = ctypes.c_void_p(0x1000)     # aligned, never dereferenced: the calls below fail before any launch
ODD = ctypes.c_void_p(0x1001)
INVALID, UNSUPPORTED, WORKSPACE = B.FASTGL_ERR_INVALID_ARG, B.FASTGL_ERR_UNSUPPORTED, B.FASTGL_ERR_WORKSPACE
NAN = float("nan")


def norm_fwd(dt=0, X=FAKE, R=None, w=FAKE, M=4, F=8, eps=1e-6, rng=None, p=0.0, s=None, Y=FAKE, rstd=None):
    return B.lib().fastgl_norm_fwd(dt, X, R, w, M, F, eps, rng, p, s, Y, rstd, None)


def norm_e4m3(dt=0, X=FAKE, w=FAKE, M=4, F=8, Q=FAKE, scale=FAKE, eps=1e-6):
    return B.lib().fastgl_norm_fwd_e4m3(dt, X, None, w, M, F, eps, None, 0.0, None, Q, scale, None, None)


def norm_bwd(dt=0, S=FAKE, w=FAKE, rstd=FAKE, dY=FAKE, dS=None, M=4, F=8, rng=None, p=0.0, dX=FAKE, dR=None, dw=None, ws=FAKE,
             wsb=1 << 30):
    return B.lib().fastgl_norm_bwd(dt, S, w, rstd, dY, dS, M, F, rng, p, dX, dR, dw, ws, wsb, None)


def dropout(dt=0, X=FAKE, R=None, M=4, F=8, rng=FAKE, p=0.5, Y=FAKE):
    return B.lib().fastgl_dropout(dt, X, R, M, F, rng, p, Y, None)


def gather(table=FAKE, scale=FAKE, rows=9, ids=FAKE, n=4, F=8, dt=0, out=FAKE):
    return B.lib().fastgl_gather_rows_e4m3(table, scale, rows, ids, n, F, dt, out, None)


@pytest.mark.parametrize("call,kw,status,text", [
    *[(f, kw, s, t) for f in (norm_fwd, norm_bwd, dropout) for kw, s, t in (
        (dict(dt=2), INVALID, "dtype"), (dict(dt=-1), INVALID, "dtype"), (dict(M=-1), INVALID, "negative"),
        (dict(F=0), INVALID, "columns"), (dict(F=-3), INVALID, "columns"), (dict(M=2 ** 31 - 1), UNSUPPORTED, "2^31"),
        (dict(F=2 ** 24 + 1), UNSUPPORTED, "2^24"), (dict(p=-0.1), INVALID, "probability"), (dict(p=1.0001), INVALID, "probability"),
        (dict(p=NAN), INVALID, "probability"), (dict(p=0.5, rng=None), INVALID, "rng"),
        (dict(p=0.5, rng=ctypes.c_void_p(0x1004)), INVALID, "rng"))],
    (norm_fwd, dict(eps=-1e-6), INVALID, "eps"), (norm_fwd, dict(eps=NAN), INVALID, "eps"),
    (norm_fwd, dict(eps=float("inf")), INVALID, "eps"), (norm_fwd, dict(X=None), INVALID, "NULL"),
    (norm_fwd, dict(w=None), INVALID, "NULL"), (norm_fwd, dict(Y=None), INVALID, "NULL"), (norm_fwd, dict(X=ODD), INVALID, "aligned"),
    (norm_fwd, dict(R=ODD), INVALID, "aligned"), (norm_fwd, dict(s=ODD), INVALID, "aligned"),
    (norm_fwd, dict(rstd=ctypes.c_void_p(0x1002)), INVALID, "aligned"), (norm_fwd, dict(dt=1, w=ctypes.c_void_p(0x1002)), INVALID, "aligned"),
    (norm_e4m3, dict(scale=None), INVALID, "NULL"), (norm_e4m3, dict(Q=None), INVALID, "NULL"),
    (norm_e4m3, dict(scale=ODD), INVALID, "aligned"), (norm_e4m3, dict(F=0), INVALID, "columns"),
    (norm_bwd, dict(S=None), INVALID, "NULL"), (norm_bwd, dict(rstd=None), INVALID, "NULL"), (norm_bwd, dict(dY=None), INVALID, "NULL"),
    (norm_bwd, dict(dS=ODD), INVALID, "aligned"), (norm_bwd, dict(dR=ODD), INVALID, "aligned"),
    (norm_bwd, dict(dw=FAKE, ws=None), INVALID, "workspace"), (norm_bwd, dict(dw=FAKE, ws=ctypes.c_void_p(0x1010)), INVALID, "workspace"),
    (norm_bwd, dict(dw=FAKE, wsb=16), WORKSPACE, "too small"), (norm_bwd, dict(dw=ODD), INVALID, "aligned"),
    (dropout, dict(X=None), INVALID, "NULL"), (dropout, dict(Y=None), INVALID, "NULL"), (dropout, dict(R=ODD), INVALID, "aligned"),
    (dropout, dict(M=2 ** 31 - 2000, F=2 ** 24), UNSUPPORTED, "one launch"),
    (gather, dict(dt=2), INVALID, "dtype"), (gather, dict(n=-1), INVALID, "negative"), (gather, dict(rows=-1), INVALID, "negative"),
    (gather, dict(F=0), INVALID, "columns"), (gather, dict(n=2 ** 31 - 1), UNSUPPORTED, "2^31"),
    (gather, dict(table=None), INVALID, "NULL"), (gather, dict(scale=None), INVALID, "NULL"), (gather, dict(ids=None), INVALID, "NULL"),
    (gather, dict(out=None), INVALID, "NULL"), (gather, dict(scale=ODD), INVALID, "aligned"),
    (gather, dict(ids=ctypes.c_void_p(0x1004)), INVALID, "aligned"), (gather, dict(out=ctypes.c_void_p(0x1002)), INVALID, "aligned"),
])
def test_bad_arguments_are_refused_before_launch(call, kw, status, text):
    assert call(**kw) == status
    assert text in B.fastgl_last_error()


def test_calls_without_rows_do_nothing():
    assert norm_fwd(M=0, X=None, Y=None) == B.FASTGL_OK and dropout(M=0, X=None, Y=None) == B.FASTGL_OK
    assert norm_bwd(M=0, S=None, rstd=None, dY=None) == B.FASTGL_OK and gather(n=0, ids=None, out=None) == B.FASTGL_OK
    assert norm_bwd(dX=None) == B.FASTGL_OK                          # nothing asked for


def test_workspace_size():
    f = B.fastgl_norm_bwd_workspace_bytes
    assert f(-1, 4) == 0 and f(4, 0) == 0 and f(0, 8) == 0
    assert f(1, 8) >= 32 and f(100_000, 256) >= 256 * 256 * 4 and f(1_000_000, 8192) <= 2048 * 8192 * 4
