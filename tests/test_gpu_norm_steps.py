"""Norm, its backward pass and gathers of so many rows that a workgroup takes several steps, on the GPU against 64 bits there."""
import numpy as np
import pytest
import torch

import rows_ref as ref
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
SENTINEL, EPS = -776.0, 1e-5


def factor(p):
    """What kept elements are multiplied by: 65536 / (65536 - t) in float32."""
    return float(np.float32(ref.drop_scale(p)))


# Every spread of a row over lanes, with rows for more than two launches' worth of groups and no multiple of a step: 1, 2, 4, ... 64 and 256
# lanes, one to four chunks a lane, and rows that are read twice.
SHAPES = [(1_100_003, 5), (600_001, 9), (600_007, 16), (300_001, 17), (300_003, 24), (300_007, 32), (140_001, 47), (70_001, 100), (140_003, 160), (40_001, 256), (70_003, 300), (17_001, 500), (20_001, 602), (17_003, 1000), (17_003, 1500),
          (4500, 2000), (4500, 2050), (4501, 5000), (2100, 8197)]


def setting(M, F, dtype, p):
    g = torch.Generator(device="cuda").manual_seed(M + F)
    t = ref.DTYPES[dtype]
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").to(t)  # noqa: E731
    rng = torch.tensor([0x1234_5678_9ABC, (1 << 40) + F], dtype=torch.int64, device="cuda")
    keep = B.fastgl_dropout(torch.ones(M, F, device="cuda"), rng, p) != 0 if p > 0 else torch.ones(M, F, dtype=torch.bool, device="cuda")
    if p > 0:                                                       # the mask itself, in the last rows
        at = np.arange(max(0, M - 3), M, dtype=np.uint64)[:, None]
        w = ref.philox(np.arange(-(-F // 8), dtype=np.uint64)[None, :], at, np.uint64(int(rng[1]) & 0xFFFFFFFF), np.uint64(int(rng[1]) >> 32),
                       int(rng[0]) & 0xFFFFFFFF, int(rng[0]) >> 32)
        halves = np.stack([h for v in w for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))], -1).reshape(at.shape[0], -1)[:, :F]
        assert torch.equal(keep[-3:].cpu(), torch.from_numpy(halves >= ref.threshold(p)))
    return make, 1.0 + 0.3 * torch.randn(F, generator=g, device="cuda"), rng, keep


def assert_within(got, want, bound, what):
    over = (got.double() - want).abs() - bound
    assert got.shape == want.shape and bool((over <= 0).all()), (what, over.max().item())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,F", SHAPES)
def test_forward_in_steps(M, F, dtype):
    t, p = ref.DTYPES[dtype], 0.4
    make, w, rng, keep = setting(M, F, dtype, p)
    x, r = make(M, F), 2 * make(M, F)
    h = torch.where(keep, x.double() * factor(p), 0.0) + r.double()
    rstd = 1.0 / torch.sqrt(h.square().mean(1) + EPS)
    y = h * rstd[:, None] * w.double()
    off_y, off_h, off_rstd = ref.norm_bounds(x, w, y, h, rstd, t, r, p)
    buf, out = ref.guarded((M, F), t, SENTINEL)
    Y, S, R = B.fastgl_norm_fwd(x, w, EPS, residual=r, rng=rng, p=p, Y=out)
    assert_within(Y, y, off_y + ref.HALF[t] * (y.abs() + off_y), "y")
    assert_within(S, h, off_h + ref.HALF[t] * (h.abs() + off_h), "h")
    assert_within(R, rstd, off_rstd, "rstd")
    assert ref.bands_intact(buf, out, SENTINEL)
    buf, q = ref.guarded((M, F), torch.float8_e4m3fn, 3.0)
    Q, scale, S8, R8 = B.fastgl_norm_fwd_e4m3(x, w, EPS, residual=r, rng=rng, p=p, Q=q)
    assert torch.equal(S8, S) and torch.equal(R8, R) and ref.bands_intact(buf, q, 3.0)
    want = (y.abs().amax(1) / 448).clamp_min(2.0 ** -126)
    assert_within(scale, want, off_y.amax(1) / 448 + 3 * ref.U32 * want, "scale")
    sc = scale.double()[:, None]
    assert_within(Q.double() * sc, y, off_y + 4 * ref.U32 * y.abs() + (2.0 ** -4 * (y.abs() + off_y) * (1 + 4 * ref.U32) + sc * 2.0 ** -10), "q")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,F", SHAPES)
def test_backward_in_steps(M, F, dtype):
    t, p = ref.DTYPES[dtype], 0.3
    make, w, rng, keep = setting(M, F, dtype, p)
    S, dY, dS = 2 * make(M, F), make(M, F), make(M, F)
    rstd = (1.0 / torch.sqrt(S.double().square().mean(1) + EPS)).float()
    bufs = [ref.guarded((M, F), t, SENTINEL) for _ in range(2)]
    gx, gr, gw = B.fastgl_norm_bwd(S, w, rstd, dY, dS=dS, rng=rng, p=p, dX=bufs[0][1], dR=bufs[1][1])
    n, tt, rs = S.double() * rstd.double()[:, None], dY.double() * w.double(), rstd.double()[:, None]
    d = rs * (tt - n * (tt * n).mean(1, keepdim=True)) + dS.double()
    mean = (tt * n).abs().mean(1, keepdim=True)
    off = ref.U32 * (rs * (4 * tt.abs() + n.abs() * ((5 + ref.chain(F) + 4) * mean)) + 2 * d.abs() + dS.double().abs()) * 1.01
    assert_within(gr, d, off + ref.HALF[t] * (d.abs() + off), "dR")
    k = factor(p)
    dx = torch.where(keep, d * k, 0.0)
    assert_within(gx, dx, (k * off + ref.U32 * dx.abs() + ref.HALF[t] * (dx.abs() + k * off)) * keep * 1.01, "dX")
    dw, size = (dY.double() * n).sum(0), (dY.double() * n).abs().sum(0)
    assert_within(gw, dw, ref.U32 * (8 + M // 256 + 10) * size, "dw")
    for buf, inner in bufs:
        assert ref.bands_intact(buf, inner, SENTINEL)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,F", SHAPES)
def test_weight_gradient_counts_every_row_once(M, F, dtype):
    """Small whole numbers, whose sums are exact in float32: the column sums are equal to the true ones."""
    g = torch.Generator(device="cuda").manual_seed(1)
    S, dY = (torch.randint(-2, 3, (M, F), generator=g, device="cuda").to(ref.DTYPES[dtype]) for _ in range(2))
    rstd = torch.ones(M, device="cuda")
    rstd[::3] = 2.0
    _, _, dw = B.fastgl_norm_bwd(S, torch.ones(F, device="cuda"), rstd, dY, want=("dw",))
    want = (S.double() * dY.double() * rstd.double()[:, None]).sum(0)
    assert 8 * M < 1 << 24 and torch.equal(dw.double(), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,F", [(M, F) for M in (1, 2, 3, 31, 64, 129) for F in (9, 15, 16, 17, 25, 32)])
def test_few_narrow_rows(M, F, dtype):
    test_forward_in_steps(M, F, dtype)
    test_backward_in_steps(M, F, dtype)
    test_weight_gradient_counts_every_row_once(M, F, dtype)


@pytest.mark.parametrize("dtype,n,F", [("bf16", 270_003, 131), ("bf16", 33_001, 1031), ("bf16", 6_800_003, 5), ("bf16", 4_300_001, 8), ("f32", 130_007, 133),
                                       ("f32", 5_700_001, 3), ("f32", 8_301, 2050), ("f32", 4_200_003, 4)])
def test_gather_of_many_rows(dtype, n, F):
    """Results of 64 MiB and more: four rows a lane.  IDs outside the table in the first and the last group."""
    rows, b = 1009, 2 if dtype == "bf16" else 4
    assert n * F * b >= 1 << 26
    g = torch.Generator(device="cuda").manual_seed(F)
    bits = torch.randint(0, 127, (rows, F), generator=g, device="cuda", dtype=torch.uint8) + 128 * torch.randint(0, 2, (rows, F), generator=g, device="cuda", dtype=torch.uint8)
    Q, scale = bits.view(torch.float8_e4m3fn), torch.rand(rows, generator=g, device="cuda") + 0.5
    ids = torch.randint(0, rows, (n,), generator=g, device="cuda")
    bad = torch.tensor([0, 7, n - 130, n - 2, n - 1], device="cuda")
    ids[bad] = torch.tensor([-1, rows, 1 << 40, -(1 << 62), rows], device="cuda")
    buf, out = ref.guarded((n, F), ref.DTYPES[dtype], SENTINEL, shift=1)
    B.fastgl_gather_rows_e4m3(Q, scale, ids, dtype, out=out)
    at = ids.clamp(0, rows - 1)
    good = torch.ones(n, dtype=torch.bool, device="cuda")
    good[bad] = False
    want = torch.where(good[:, None], Q.float()[at] * scale[at][:, None], float("nan")).to(ref.DTYPES[dtype])      # one product, one rounding
    assert torch.equal(torch.isnan(out), ~good[:, None].expand(n, F)) and torch.equal(out[good], want[good])
    assert ref.bands_intact(buf, out, SENTINEL)
