"""The loss's plain form on the CPU: gradients against differences, and what the entry points refuse."""
import ctypes

import pytest
import torch

from loss_ref import Loss
from paper_2409_14939_amd import binding as B


def test_gradients_against_differences():
    g = torch.Generator().manual_seed(1)
    H, W, b = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((6, 4), (4, 5), (5,)))
    label, dloss = torch.tensor([0, 4, -1, 2, 2, -7]), torch.rand(6, generator=g, dtype=torch.float64)
    ref = Loss(H, W, b, label).backward(dloss)
    for x, grad in ((H, ref.dH), (W, ref.dW), (b, ref.db)):
        flat, want = x.view(-1), grad.reshape(-1)
        for i in range(flat.numel()):
            keep, values = flat[i].item(), []
            for step in (1e-6, -1e-6):
                flat[i] = keep + step
                values.append((Loss(H, W, b, label).loss * dloss).sum().item())
            flat[i] = keep
            assert abs((values[0] - values[1]) / 2e-6 - want[i].item()) < 1e-8


def test_a_row_by_hand():
    ref = Loss(torch.tensor([[1.0]]), torch.tensor([[0.0, 0.0, 0.0]]), torch.log(torch.tensor([1.0, 2.0, 5.0])), torch.tensor([1]))
    assert abs(ref.loss.item() - torch.log(torch.tensor(4.0)).item()) < 1e-6
    ref.backward(torch.tensor([8.0]))
    assert torch.allclose(ref.db, torch.tensor([1.0, -6.0, 5.0], dtype=torch.float64), atol=1e-6)


FAKE, ODD, TWO, FOUR = (ctypes.c_void_p(x) for x in (0x1000, 0x1001, 0x1002, 0x1004))
INVALID, UNSUPPORTED, WORKSPACE = B.FASTGL_ERR_INVALID_ARG, B.FASTGL_ERR_UNSUPPORTED, B.FASTGL_ERR_WORKSPACE


def fwd(dt=1, H=FAKE, W=FAKE, b=None, label=FAKE, M=64, K=8, N=512, loss=FAKE, lse=FAKE, ws=FAKE, wsb=1 << 50):
    return B.lib().fastgl_loss_fwd(dt, H, W, b, label, M, K, N, loss, lse, ws, wsb, None)


def bwd(dt=1, H=FAKE, W=FAKE, b=None, label=FAKE, lse=FAKE, dloss=FAKE, M=64, K=8, N=512, dH=FAKE, dW=FAKE, db=FAKE, ws=FAKE, wsb=1 << 50):
    return B.lib().fastgl_loss_bwd(dt, H, W, b, label, lse, dloss, M, K, N, dH, dW, db, ws, wsb, None)


@pytest.mark.parametrize("call,kw,status,text", [
    *[(f, kw, s, t) for f in (fwd, bwd) for kw, s, t in (
        (dict(dt=2), INVALID, "dtype"), (dict(M=-1), INVALID, "negative"), (dict(K=-1), INVALID, "negative"), (dict(N=-1), INVALID, "negative"),
        (dict(N=0), INVALID, "classes"), (dict(M=2 ** 31 - 1), UNSUPPORTED, "2^31"), (dict(K=2 ** 20 + 1), UNSUPPORTED, "2^20"),
        (dict(N=2 ** 21 + 1), UNSUPPORTED, "2^21"), (dict(H=None), INVALID, "NULL"), (dict(W=None), INVALID, "NULL"), (dict(label=None), INVALID, "NULL"),
        (dict(H=ODD), INVALID, "aligned"), (dict(dt=0, W=TWO), INVALID, "aligned"), (dict(b=TWO), INVALID, "aligned"), (dict(label=FOUR), INVALID, "aligned"),
        (dict(lse=TWO), INVALID, "aligned"), (dict(ws=None), INVALID, "workspace"), (dict(ws=ctypes.c_void_p(0x1010)), INVALID, "workspace"),
        (dict(wsb=64), WORKSPACE, "too small"))],
    (fwd, dict(loss=None), INVALID, "NULL"), (fwd, dict(loss=TWO), INVALID, "aligned"),
    (bwd, dict(lse=None), INVALID, "NULL"), (bwd, dict(dloss=None), INVALID, "NULL"), (bwd, dict(dloss=TWO), INVALID, "aligned"),
    (bwd, dict(dH=ODD), INVALID, "aligned"), (bwd, dict(dW=ODD), INVALID, "aligned"), (bwd, dict(db=TWO), INVALID, "aligned")])
def test_bad_arguments_are_refused_before_launch(call, kw, status, text):
    assert call(**kw) == status
    assert text in B.fastgl_last_error()


def test_calls_with_nothing_to_do():
    assert fwd(M=0, H=None, label=None, loss=None) == B.FASTGL_OK and fwd(M=0, N=0) == B.FASTGL_OK
    assert bwd(dH=None, dW=None, db=None, H=None, label=None) == B.FASTGL_OK


def test_workspace_sizes():
    f, b = B.fastgl_loss_fwd_workspace_bytes, B.fastgl_loss_bwd_workspace_bytes
    assert f("bf16", 0, 8, 8) == 0 and f("bf16", 8, -1, 8) == 0 and b("f32", 8, 8, 0) == 0 and b("bf16", 8, 8, 2 ** 22) == 0
    for dt in ("f32", "bf16"):
        for M, K, N in ((1, 8, 500), (8000, 256, 470), (8192, 512, 65_536), (1000, 4096, 2 ** 21), (2 ** 21, 64, 200), (2 ** 22, 64, 200)):
            assert f(dt, M, K, N) >= f(dt, M, K, N, True) and b(dt, M, K, N) >= b(dt, M, K, N, True)
            # a piece of dZ and one of the weights, H, sums; never M N or K N
            rows = (M + 255) // 256 * 256
            least = 6 * rows * 256 + (1 << 30) + (1 << 30) + 6 * K * 512 + 6 * M * (K + 8)
            assert b(dt, M, K, N) < least + 64 * 4 * max(M * K, K * 4096) + (1 << 28)
            assert f(dt, M, K, N) < (1 << 30) + 6 * K * 512 + 6 * M * (K + 8) + 4 * M + 8 * M * (N // 64 + 300) + (1 << 20)
