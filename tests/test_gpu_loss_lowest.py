"""Class scores at the ends of float32: a bias of the type's lowest value rules a class out, and what lies beyond 2^128 / log2 e."""
import pytest
import torch

from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
LOWEST = torch.finfo(torch.float32).min
SIZES = [(7, 5, 47), (80, 8, 700), (4000, 8, 3000), (2000, 200, 2500)]            # one strip of classes, several; tiles forward, and both ways


def inputs(M, K, N, dtype):
    g = torch.Generator(device="cuda").manual_seed(N)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")
    H, W = make(M, K).to(dtype), make(K, N).to(dtype)
    return H, W, make(N), torch.randint(0, N, (M,), generator=g, device="cuda"), make(M)


def step(H, W, b, label, dloss):
    loss, lse = B.fastgl_loss_fwd(H, W, b, label)
    return [loss, lse, *B.fastgl_loss_bwd(H, W, b, label, lse, dloss)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_the_lowest_value_rules_a_class_out_as_minus_infinity_does(M, K, N, dtype):
    """Runs of classes as wide as a tile and more, and single ones: the same bits."""
    H, W, b, label, dloss = inputs(M, K, N, dtype)
    out = torch.arange(N, device="cuda") % 5 == 2
    out[N // 10:N // 2] = True
    label[out[label]] = 0
    assert not bool(out[0])
    results = []
    for low in (LOWEST, -float("inf"), -2.5e38):               # the last: below what log2 e times it can be
        b[out] = low
        results.append(step(H, W, b, label, dloss))
    for got in results:
        assert all(bool(torch.isfinite(x).all()) for x in got)
    for i, (a, b_, c) in enumerate(zip(*results)):
        assert torch.equal(a, b_) and torch.equal(a, c), i
    assert not bool(results[0][4][out].any()) and not bool(results[0][3][:, out].any())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("low", [LOWEST, -2.5e38, 3e38])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_scores_whose_logarithm_of_two_is_no_float(M, K, N, low, dtype):
    """All classes at one such value, which swallows everything else: lse is that value, every weight exp(0) = 1."""
    H, W, b, label, dloss = inputs(M, K, N, dtype)
    b[:] = low
    label[1::3] = -1
    loss, lse, dH, dW, db = step(H, W, b, label, dloss)
    assert bool((lse == b[0]).all()) and not bool(loss.any())
    dz = dloss[:, None].double().repeat(1, N)
    dz[torch.arange(M, device="cuda"), label.clamp(min=0)] = 0
    dz[1::3] = 0
    # sums of M float32 terms, in any order
    assert bool(((db - dz.sum(0)).abs() <= 2.0 ** -24 * (M + 8) * dz.abs().sum(0)).all()) and bool(torch.isfinite(dH).all()) and bool(torch.isfinite(dW).all())
    # one class far above the others takes all the weight
    b.normal_()
    b[3] = abs(low)
    if abs(low) < 3.3e38:
        loss, lse, dH, dW, db = step(H, W, b, torch.full_like(label, 3), dloss)
        assert bool((lse == b[3]).all()) and not any(bool(x.any()) for x in (loss, dH, dW, db))
