"""The operators of a residual feed-forward block on arrays of more than 2^31 elements: rows on both sides of where an offset of 31
or 32 bits ends, against 64 bits."""
import pytest
import torch

import gated_ref
import rows_ref as ref
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-5


def rows_around(M, F):
    """The first and last rows, and those around 2^30, 2^31 and 2^32 elements (2^31 and 2^32 bytes of bf16 among them)."""
    at = {0, 1, M - 2, M - 1}
    for e in (30, 31, 32):
        at |= {r for r in range((1 << e) // F - 2, (1 << e) // F + 3) if 0 <= r < M}
    return torch.tensor(sorted(at), device="cuda")


def filled(M, F, seed):
    """bfloat16 [M, F]: a period of rows of random values, so that no larger type of it exists."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    period = torch.randn(9973, F, generator=g, device="cuda").bfloat16()
    return period.repeat(-(-M // 9973), 1)[:M]


def assert_within(got, want, bound, what):
    over = (got.double() - want).abs() - bound
    assert bool((over <= 0).all()), (what, over.max().item())


def test_norm_dropout_and_gather():
    F = 1030
    M, half = (1 << 32) // F + 40, 2.0 ** -8
    x, w = filled(M, F, 1), 1.0 + 0.3 * torch.randn(F, generator=torch.Generator().manual_seed(2)).cuda()
    at = rows_around(M, F)
    y, _, rstd = B.fastgl_norm_fwd(x, w, EPS)
    want, _, want_rstd = ref.norm(x[at], w, EPS)
    off_y, _, off_rstd = ref.norm_bounds(x[at], w, want, x[at].double(), want_rstd, torch.bfloat16)
    assert_within(y[at], want, off_y + half * (want.abs() + off_y), "y")
    assert_within(rstd[at], want_rstd, off_rstd, "rstd")
    # backward, with y as the gradient
    dX, _, _ = B.fastgl_norm_bwd(x, w, rstd, y, want=("dX",))
    n, t, rs = x[at].double() * rstd[at].double()[:, None], y[at].double() * w.double(), rstd[at].double()[:, None]
    d, mean = rs * (t - n * (t * n).mean(1, keepdim=True)), (t * n).abs().mean(1, keepdim=True)
    off = ref.U32 * (rs * (4 * t.abs() + n.abs() * ((9 + ref.chain(F)) * mean)) + 2 * d.abs()) * 1.01
    assert_within(dX[at], d, off + half * (d.abs() + off), "dX")
    del dX, y
    # 8-bit rows, and all of them gathered from that table in the other order
    Q, scale, _, _ = B.fastgl_norm_fwd_e4m3(x, w, EPS, want_rstd=False)
    ids = torch.arange(M - 1, -1, -1, device="cuda")
    rows = B.fastgl_gather_rows_e4m3(Q, scale, ids, "bf16")
    assert torch.equal(rows[at], (Q[ids[at]].float() * scale[ids[at]][:, None]).bfloat16())
    bound = off_y + 4 * ref.U32 * want.abs() + 2.0 ** -4 * (want.abs() + off_y) * (1 + 4 * ref.U32) + scale[at].double()[:, None] * 2.0 ** -10
    assert_within(Q[at].double() * scale[at].double()[:, None], want, bound, "q")
    del rows, Q
    # dropout: the mask of a row does not depend on the rows before it
    rng = torch.tensor([123, 1 << 40], dtype=torch.int64, device="cuda")
    z = B.fastgl_dropout(x, rng, 0.5)
    for r in at.tolist():
        keep = ref_keep_row(r, F, 0.5, rng.tolist())
        assert torch.equal(z[r].cpu(), torch.where(keep, 2 * x[r].cpu(), torch.zeros((), dtype=torch.bfloat16)))


def ref_keep_row(row, F, p, state):
    import numpy as np
    blocks = -(-F // 8)
    w = ref.philox(np.arange(blocks, dtype=np.uint64), np.uint64(row), np.uint64(state[1] & 0xFFFFFFFF), np.uint64(state[1] >> 32),
                   state[0] & 0xFFFFFFFF, state[0] >> 32)
    halves = np.stack([h for v in w for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))], -1).reshape(blocks * 8)
    return torch.from_numpy(halves[:F] >= ref.threshold(p))


def test_gated():
    M, K, N = 1_060_000, 24, 4072                                  # 2^32 elements of G and more, in blocks of columns
    assert M * N > (1 << 32)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = filled(M, K, 4)
    wg, wu = (torch.randn(K, N, generator=g, device="cuda").bfloat16() / 4 for _ in range(2))
    at = rows_around(M, N)
    P, G, U = B.fastgl_gated_fwd(x, wg, wu, None, None, "relu")
    xd = x[at].double()
    u = xd @ wu.double()
    size = xd.abs() @ wg.double().abs() + xd.abs() @ wu.double().abs()
    off = size * gated_ref.U32 * 1.3 * (K + 4)
    gd = xd @ wg.double()
    assert_within(G[at], gd, off + 2.0 ** -8 * (gd.abs() + off), "G")
    assert_within(U[at], u, off + 2.0 ** -8 * (u.abs() + off), "U")
    p, off_p = gd.clamp_min(0) * u, off * (u.abs() + gd.abs() + off)
    assert_within(P[at], p, off_p + 2.0 ** -8 * (p.abs() + off_p) + 1e-37, "P")
    del P
    # gradients: whole numbers in the chosen rows and 0 elsewhere, so that the weights' are exact
    G.fill_(1.0)
    U.fill_(1.0)
    dP = torch.zeros(M, N, device="cuda", dtype=torch.bfloat16)
    dP[at] = torch.randint(-2, 3, (at.numel(), N), generator=g, device="cuda").bfloat16()
    ones = torch.ones(M, K, device="cuda", dtype=torch.bfloat16)
    ones[at] = torch.randint(-2, 3, (at.numel(), K), generator=g, device="cuda").bfloat16()
    wg, wu = (torch.randint(-1, 2, (K, N), generator=g, device="cuda").bfloat16() for _ in range(2))
    dX, dWg, dWu, dbg, dbu = B.fastgl_gated_bwd(ones, wg, wu, G, U, dP, "relu")
    want = ones[at].double().t() @ dP[at].double()
    assert torch.equal(dWg.double(), want) and torch.equal(dWu.double(), want)
    assert torch.equal(dbg.double(), dP[at].double().sum(0)) and torch.equal(dbu, dbg)
    assert torch.equal(dX[at], (dP[at].double() @ (wg.double() + wu.double()).t()).bfloat16())
    rest = torch.ones(M, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert bool((dX[rest] == 0).all())
