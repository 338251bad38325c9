"""Large calls of the loss with few terms that are not 0, spread over all of a sum: bounds that wrong offsets, missing rows and results of 0 pass by far."""
import pytest
import torch

from loss_ref import HALF, Loss
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def spread(n, count, seed):
    """Indices from the first to the last, those around multiples of 32, 256 and powers of two among them."""
    g = torch.Generator().manual_seed(seed)
    edges = [x + d for x in (32, 256, 1 << 14, n // 2 // 256 * 256, n // 256 * 256, 1 << 21) for d in (-1, 0, 1)]
    some = torch.cat((torch.tensor([0, n - 1] + [x for x in edges if 0 <= x < n]), torch.randint(0, n, (count,), generator=g)))
    return some.unique().cuda()


def compare(got, want, off, t, what):
    bad = (got.double() - want).abs() > off + HALF[t] * (want.abs() + off)
    assert not bool(bad.any()), (what, int(bad.sum()))
    # zeros, and neighbours' results in the place of these, would not pass
    assert float((want.abs() > 4 * off).double().mean()) > 0.7, what
    rolled = want.roll(1, 0)
    assert float(((rolled - want).abs() > off + HALF[t] * (want.abs() + off)).double().mean()) > 0.7, what


@pytest.mark.parametrize("coarse", [False, True])
@pytest.mark.parametrize("dtype,M,K,N", [("f32", 300, 60_000, 3100), ("bf16", 64, 200_000, 2801)])
def test_many_inputs_with_packed_weights_in_pieces(dtype, M, K, N, coarse):
    """Sixty inputs that are not 0; results are compared there and at as many others."""
    t = DTYPES[dtype]
    planes = 3 if dtype == "f32" else 1
    assert 2 * planes * K * N > 1 << 30
    g = torch.Generator(device="cuda").manual_seed(8)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")
    W = (0.5 * make(K, N)).to(t)
    inputs, others = spread(K, 45, 1), spread(K, 60, 2)
    H = torch.zeros(M, K, device="cuda", dtype=t)
    H[:, inputs] = make(M, len(inputs)).to(t)
    b, dloss, label = 0.5 * make(N), 1.0 + torch.rand(M, generator=g, device="cuda"), torch.randint(-1, N, (M,), generator=g, device="cuda")
    loss, lse = B.fastgl_loss_fwd(H, W, b, label)
    dH, dW, db = B.fastgl_loss_bwd(H, W, b, label, lse, dloss, coarse=coarse)
    at = torch.cat((inputs, others)).unique()
    ref = Loss(H[:, at], W[at], b, label).backward(dloss)
    on = label >= 0
    compare(loss[on], ref.loss[on], ref.off_loss[on], torch.float32, "loss")
    compare(lse, ref.lse, ref.off_lse, torch.float32, "lse")
    compare(dH[:, at][on], ref.dH[on], ref.off_dH[on], t, "dH")
    k = torch.isin(at, inputs)
    compare(dW[at[k]].T, ref.dW[k].T, ref.off_dW[k].T, t, "dW")
    compare(db, ref.db, ref.off_db, torch.float32, "db")
    rest = torch.ones(K, dtype=torch.bool, device="cuda")
    rest[inputs] = False
    assert not bool(dW[rest].any()) and not bool(dH[~on].any())


@pytest.mark.parametrize("coarse", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [((1 << 21) + 300, 9, 12), ((1 << 21) + 1, 64, 40), ((1 << 21) + 77, 24, 300), ((1 << 22) + 130, 17, 47), (1 << 21, 40, 100),
                                   (400_000, 9, 9000)])
def test_many_rows_few_of_which_have_a_label(dtype, M, K, N, coarse):
    """dZ in blocks of 32 columns up to 2^21 rows, in whole rows beyond; one piece of the classes and several."""
    t = DTYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(9)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")
    H, W, b = make(M, K).to(t), (2.0 * make(K, N) / K ** 0.5).to(t), 0.5 * make(N)
    on = spread(M, 300, 3)
    label = torch.full((M,), -1, device="cuda", dtype=torch.int64)
    label[on] = torch.randint(0, min(N, 200), (len(on),), generator=g, device="cuda") * (N // min(N, 200))
    dloss = make(M)
    loss, lse = B.fastgl_loss_fwd(H, W, b, label)
    dH, dW, db = B.fastgl_loss_bwd(H, W, b, label, lse, dloss, coarse=coarse)
    ref = Loss(H[on], W, b, label[on]).backward(dloss[on])
    compare(loss[on], ref.loss, ref.off_loss, torch.float32, "loss")
    compare(dH[on], ref.dH, ref.off_dH, t, "dH")
    hit = torch.zeros(N, dtype=torch.bool, device="cuda")           # classes that are a label: those of no row hold weights of some thousandth alone
    hit[label[on]] = True
    compare(dW.T[hit], ref.dW.T[hit], ref.off_dW.T[hit], t, "dW")
    compare(db[hit], ref.db[hit], ref.off_db[hit], torch.float32, "db")
    for got, want, off, kind in ((dW, ref.dW, ref.off_dW, t), (db, ref.db, ref.off_db, torch.float32)):
        assert bool(((got.double() - want).abs() <= off + HALF[kind] * (want.abs() + off)).all())
    rest = torch.ones(M, dtype=torch.bool, device="cuda")
    rest[on] = False
    assert not bool(dH[rest].any()) and not bool(loss[rest].any())
