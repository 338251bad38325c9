"""How far the loss's backward pass keeps dZ for its two products: two bf16 pieces in bf16 calls, one where the caller asks for it, at every size."""
import pytest
import torch

import rows_ref
from loss_ref import HALF, U32, Loss
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = rows_ref.DTYPES
# rows, classes: calls of the kernel of small ones, and of the tiles; several pieces of the classes
SIZES = [(1, 9), (64, 47), (300, 65), (4096, 4096), (513, 9001), (9000, 33_000)]


def exact_inputs(M, N, dtype, seed=0):
    """Scores of 256 for one class of each row and 0 for the others: dZ is dloss there, -dloss at the label and 0 elsewhere, to the bit.
    dloss has 16 bits, which two bf16 hold; H and W are small whole numbers, so that sums of some hundred products are exact in float32."""
    g = torch.Generator().manual_seed(seed)
    tops = min(4, N - 1)
    H, W = torch.zeros(M, 24), torch.zeros(24, N)
    which, tall = torch.arange(M) % tops, torch.randperm(N, generator=g)[:tops]
    H[torch.arange(M), which] = 1.0
    W[torch.arange(tops), tall] = 256.0
    H[:, 4:12] = torch.randint(-1, 2, (M, 8), generator=g).float()
    W[12:] = torch.randint(-7, 8, (12, N), generator=g).float()
    label = torch.full((M,), -1)
    on = torch.linspace(0, M - 1, min(M, 120)).long().unique()                # from the first row to the last
    label[on] = torch.randint(0, N, (len(on),), generator=g)
    label = torch.where(label == tall[which], (label + 1) % N, label)
    dloss = torch.randint(1 << 15, 1 << 16, (M,), generator=g).float() / (1 << 15)
    return H.to(dtype), W.to(dtype), label, dloss, tall[which]


@pytest.mark.parametrize("dtype,coarse", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
@pytest.mark.parametrize("M,N", SIZES)
def test_the_terms_are_kept_by_one_rule_at_all_sizes(M, N, dtype, coarse):
    H, W, label, dloss, top = (x.cuda() for x in exact_inputs(M, N, DTYPES[dtype]))
    lse = torch.full((M,), 256.0, device="cuda")
    on = torch.nonzero(label >= 0)[:, 0]
    g = dloss[on]
    rounded = g.bfloat16() if coarse and dtype == "bf16" else g
    assert M < 64 or not torch.equal(g.bfloat16().float(), g)
    dz = torch.zeros(len(on), N, dtype=torch.float64, device="cuda")
    row = torch.arange(len(on), device="cuda")
    dz[row, top[on]], dz[row, label[on]] = rounded.double(), -rounded.double()
    dH, dW, db = B.fastgl_loss_bwd(H, W, None, label, lse, dloss, want=("dH", "dW", "db"), coarse=coarse)
    want = torch.zeros(M, 24, dtype=torch.float64, device="cuda")
    want[on] = dz @ W.double().T
    for got, exact, what in ((dH, want, "dH"), (dW, H[on].double().T @ dz, "dW")):
        assert torch.equal(exact.float().double(), exact), what
        bad = got != exact.to(got.dtype)
        assert not bool(bad.any()), (what, int(bad.sum()), got[bad][:4], exact[bad][:4])
    dz[row, top[on]], dz[row, label[on]] = g.double(), -g.double()             # column sums are of the unrounded terms
    assert torch.equal(db.double(), dz.sum(0))


def cancelling_inputs(M, N, dtype, seed):
    """Rows in pairs of opposite sign and nearly the same dloss, in columns of H that no score goes by; classes in pairs of opposite sign and
    nearly the same bias, in rows of W that no row takes: what remains of dH and dW there is 2^-11 of its terms."""
    g = torch.Generator().manual_seed(seed)
    make = lambda *s: torch.randn(*s, generator=g)
    H, W = torch.zeros(M, 16), torch.zeros(16, N)
    H[:, :8], W[:8] = make((M + 1) // 2, 8).repeat_interleave(2, 0)[:M], make(8, (N + 1) // 2).repeat_interleave(2, 1)[:, :N] / 8 ** 0.5
    sign = lambda n: torch.where(torch.arange(n) % 2 == 0, 1.0, -1.0)
    H[:, 8:12], W[12:] = sign(M)[:, None], sign(N)
    b = 0.5 * make((N + 1) // 2).repeat_interleave(2)[:N] + 2.0 ** -11 * (torch.arange(N) % 2)
    dloss = (0.5 + torch.rand((M + 1) // 2, generator=g)).repeat_interleave(2)[:M] * (1 + 2.0 ** -11 * (torch.arange(M) % 2))
    label = torch.randint(0, N, ((M + 1) // 2,), generator=g).repeat_interleave(2)[:M]
    out = torch.ones(M // 2, dtype=torch.bool)
    out[torch.linspace(0, M // 2 - 1, min(M // 2, 150)).long()] = False        # most pairs of a large call have no label
    label[:2 * (M // 2)][out.repeat_interleave(2)] = -1
    return H.to(dtype), W.to(dtype), b, label, dloss


@pytest.mark.parametrize("M,N", [(64, 48), (400, 600), (4096, 4096), (600, 9000)])
def test_what_remains_of_terms_that_cancel(M, N):
    H, W, b, label, dloss = (x.cuda() for x in cancelling_inputs(M, N, torch.bfloat16, seed=M))
    on = label >= 0
    ref = Loss(H[on], W, b, label[on]).backward(dloss[on])
    lse = B.fastgl_loss_fwd(H, W, b, label)[1]
    dH, dW, _ = B.fastgl_loss_bwd(H, W, b, label, lse, dloss)
    assert not bool(dH[~on].any())
    # the bound of Loss with 2^-17 in the place of a bf16's rounding of dZ
    hot = torch.zeros_like(ref.p)
    hot[torch.arange(len(hot)), label[on]] = 1.0
    size = dloss[on].double()[:, None] * (ref.p - hot).abs()
    less = HALF[torch.bfloat16] - 2.0 ** -17
    for got, want, off, terms, part in ((dH[on], ref.dH, ref.off_dH, size @ W.double().T.abs(), slice(12, 16)),
                                        (dW.T, ref.dW.T, ref.off_dW.T, (H[on].double().T.abs() @ size).T, slice(8, 12))):
        bound = (off - less * terms)[:, part]
        want = want[:, part]
        assert bool(((got[:, part].double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound)).all())
    # the check can fail: half of what remains is more than the bound allows, for most of the weights' gradients
    want, off = ref.dW[8:12], (ref.off_dW - less * (H[on].double().T.abs() @ size))[8:12]
    assert bool((off < want.abs() / 4).double().mean() > 0.5), (off.median().item(), want.abs().median().item())


def test_fp32_calls_know_one_rule():
    g = torch.Generator(device="cuda").manual_seed(3)
    for M, K, N in ((70, 40, 47), (3000, 200, 1500)):
        H, W = torch.randn(M, K, generator=g, device="cuda"), torch.randn(K, N, generator=g, device="cuda") / K ** 0.5
        label, dloss = torch.randint(-1, N, (M,), generator=g, device="cuda"), torch.rand(M, generator=g, device="cuda")
        lse = B.fastgl_loss_fwd(H, W, None, label)[1]
        for a, b in zip(B.fastgl_loss_bwd(H, W, None, label, lse, dloss), B.fastgl_loss_bwd(H, W, None, label, lse, dloss, coarse=True)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, 256, 47), (129, 200, 48), (513, 48, 700), (2100, 520, 264), (40, 33, 5000)])
def test_the_coarse_pass_stays_within_its_rounding(M, K, N, dtype):
    g = torch.Generator().manual_seed(M)
    H, W = torch.randn(M, K, generator=g).to(DTYPES[dtype]), (2.0 * torch.randn(K, N, generator=g) / K ** 0.5).to(DTYPES[dtype])
    b, label, dloss = 0.5 * torch.randn(N, generator=g), torch.randint(-1, N, (M,), generator=g), (0.5 + torch.rand(M, generator=g)) / M
    ref = Loss(H, W, b, label).backward(dloss)
    H, W, b, label, dloss = (x.cuda() for x in (H, W, b, label, dloss))
    lse = B.fastgl_loss_fwd(H, W, b, label)[1]
    need = B.fastgl_loss_bwd_workspace_bytes(dtype, M, K, N, True, coarse=True)
    ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    grads = B.fastgl_loss_bwd(H, W, b, label, lse, dloss, workspace=ws[:need], coarse=True)
    assert bool((ws[need:] == 0xA5).all())
    for got, name, t in zip(grads, ("dH", "dW", "db"), (H.dtype, H.dtype, torch.float32)):
        want, off = getattr(ref, name), getattr(ref, "off_" + name)
        assert bool(((got.double().cpu() - want).abs() <= off + HALF[t] * (want.abs() + off)).all()), name
