"""Rows without a label, and the rows that fill a tile, add nothing to the gradients whatever the weights and the bias hold."""
import pytest
import torch

from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,K,N", [(7, 5, 47), (80, 8, 700), (4000, 8, 3000), (2001, 200, 2500)])
def test_what_weights_and_bias_hold_reaches_no_gradient_of_such_rows(M, K, N, dtype):
    g = torch.Generator(device="cuda").manual_seed(N)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")
    H, W, b, label, dloss = make(M, K).to(dtype), make(K, N).to(dtype), make(N), torch.randint(0, N, (M,), generator=g, device="cuda"), make(M)
    # a class that infinite weights rule out for every row with a label: their sums of products are -inf, 0 times -inf of the others' is NaN
    H[:, 0] = H[:, 0].abs() + 0.5
    # (float32 products come from three bf16 pieces, and those of an infinity are inf, inf - inf = NaN and NaN: such a score is NaN by the
    # arithmetic that the header states, for every row, and only the small calls' own products know infinite weights)
    W[0, N // 2] = -float("inf") if dtype is torch.bfloat16 or M < 100 else -1e38
    label[label == N // 2] = 0
    label[2::3] = -1
    H[2::3, 0] = 0
    on = label >= 0
    loss, lse = B.fastgl_loss_fwd(H, W, b, label)
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(lse[on]).all())
    _, dW, db = B.fastgl_loss_bwd(H, W, b, label, lse, dloss, want=("dW", "db"))
    assert bool(torch.isfinite(dW).all()) and bool(torch.isfinite(db).all()) and not bool(dW[:, N // 2].any()) and db[N // 2] == 0
    # a batch without any label: a bias of NaN and infinities reaches nothing
    W[0, N // 2] = 1.0
    b[::3], b[1::3] = float("nan"), float("inf")
    none = torch.full_like(label, -1)
    loss, lse = B.fastgl_loss_fwd(H, W, b, none)
    for x in (loss, *B.fastgl_loss_bwd(H, W, b, none, lse, dloss)):
        assert not bool(x.any())
