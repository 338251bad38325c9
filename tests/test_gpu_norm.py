"""Norm, dropout and e4m3 rows on the GPU against their plain 64-bit forms (tests/rows_ref.py)."""
import numpy as np
import pytest
import torch

import rows_ref as ref
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
SENTINEL = -776.0                  # of either type
WIDTHS = [1, 2, 7, 8, 9, 47, 64, 65, 100, 128, 131, 256, 257, 512, 602, 1000, 1024, 1031, 2048, 2050, 4096, 4099, 8192, 8197, 20_003]
EPS = 1e-5


def rows_for(F):
    return 37 if F > 2048 else 133


def make(M, F, dtype, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(M, F, generator=g)).to(ref.DTYPES[dtype])


def state(seed=0):
    return torch.tensor([0x1234_5678_9ABC + seed, (1 << 40) + 12345 + seed], dtype=torch.int64, device="cuda")


def assert_within(got, want, bound, what):
    got, want = got.double().cpu(), want.double()
    assert got.shape == want.shape, what
    over = (got - want).abs() - bound
    assert bool(torch.isfinite(got).all()) and bool((over <= 0).all()), (what, over.max().item(), (got - want).abs().max().item())


# --------------------------------------------------------------------------------- dropout
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", [1, 3, 8, 9, 47, 100, 256, 1000, 8191, 16_384, 16_400, 40_001])
def test_dropout(F, dtype):
    M = max(3, 60_000 // F)
    x, r = make(M, F, dtype, 1), make(M, F, dtype, 2)
    s, t = state(F), ref.DTYPES[dtype]
    for p, res in ((0.0, None), (0.1, None), (0.5, r), (1.0, r)):
        buf, out = ref.guarded((M, F), t, SENTINEL, shift=1)
        B.fastgl_dropout(ref.shifted(x), s if p else None, p, residual=None if res is None else ref.shifted(res, 3), out=out)
        d = ref.drop(x.double(), p, s.tolist())
        want = d if res is None else d + res.double()
        # the product, the sum and the result's type: a rounding each
        bound = 1.01 * (ref.U32 * (d.abs() + want.abs()) + ref.HALF[t] * want.abs()) + (2.0 ** -140 if dtype == "bf16" else 0.0)
        assert_within(out, want, bound, (F, p))
        assert ref.bands_intact(buf, out, SENTINEL)
        if p and res is None:
            assert torch.equal(out.cpu() != 0, ref.keep(M, F, p, s.tolist()) & (x != 0))


def test_dropout_of_what_is_not_finite_and_at_the_ends():
    x = torch.full((64, 40), float("nan"))
    x[1::2] = float("inf")
    s = state()
    y = B.fastgl_dropout(x.cuda(), s, 0.5).cpu()
    k = ref.keep(64, 40, 0.5, s.tolist())
    assert bool((y[~k] == 0).all()) and bool(torch.isnan(y[0::2][k[0::2]]).all()) and bool(torch.isinf(y[1::2][k[1::2]]).all())
    assert bool((B.fastgl_dropout(x.cuda(), s, 1.0) == 0).all())
    for M, F in ((0, 7), (1, 1)):
        assert B.fastgl_dropout(torch.ones(M, F).cuda(), s, 0.5).shape == (M, F)


def test_dropout_of_very_many_rows():
    M, F = 9_000_001, 1                                     # a chunk a row; many workgroups
    x = torch.ones(M, F, device="cuda", dtype=torch.bfloat16)
    s = state(5)
    y = B.fastgl_dropout(x, s, 0.5).cpu().view(-1)
    at = np.r_[0:1000, 4_000_000:4_001_000, M - 1000:M]
    w = ref.philox(np.uint64(0), at.astype(np.uint64), np.uint64(int(s[1]) & 0xFFFFFFFF), np.uint64(int(s[1]) >> 32),
                   int(s[0]) & 0xFFFFFFFF, int(s[0]) >> 32)
    assert torch.equal(y[at] != 0, torch.from_numpy((w[0] & np.uint64(0xFFFF)) >= ref.threshold(0.5)))


# --------------------------------------------------------------------------------- forward
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", WIDTHS)
def test_norm_forward(F, dtype):
    M, t = rows_for(F), ref.DTYPES[dtype]
    x, r, w = make(M, F, dtype, 1), make(M, F, dtype, 2, 2.0), 1.0 + 0.3 * make(1, F, "f32", 3)[0]
    s = state(F)
    for p, res in ((0.0, None), (0.0, r), (0.3, None), (0.5, r)):
        y, h, rstd = ref.norm(x, w, EPS, res, p, s.tolist())
        off_y, off_h, off_rstd = ref.norm_bounds(x, w, y, h, rstd, t, res, p)
        bufs = [ref.guarded((M, F), t, SENTINEL, shift=1), ref.guarded((M, F), t, SENTINEL, shift=3), ref.guarded((M,), torch.float32, SENTINEL)]
        with_sum = res is not None or p > 0
        Y, S, R = B.fastgl_norm_fwd(ref.shifted(x), ref.shifted(w), EPS, residual=None if res is None else ref.shifted(res, 3), rng=s, p=p,
                                    Y=bufs[0][1], sum_out=bufs[1][1] if with_sum else None, rstd=bufs[2][1])
        assert_within(Y, y, off_y + ref.HALF[t] * (y.abs() + off_y), (F, p, "y"))
        assert_within(R, rstd, off_rstd, (F, p, "rstd"))
        assert (S is None) == (not with_sum)
        if with_sum:
            assert_within(S, h, off_h + ref.HALF[t] * (h.abs() + off_h), (F, p, "h"))
        for buf, inner in bufs:
            if inner is not bufs[1][1] or with_sum:
                assert ref.bands_intact(buf, inner, SENTINEL)
        # fewer results asked for: the same values
        Y2, S2, R2 = B.fastgl_norm_fwd(x.cuda(), w.cuda(), EPS, residual=None if res is None else res.cuda(), rng=s, p=p,
                                       want_sum=False, want_rstd=False)
        assert S2 is None and R2 is None and torch.equal(Y, Y2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", WIDTHS)
def test_norm_to_e4m3(F, dtype):
    M, t = rows_for(F), ref.DTYPES[dtype]
    x, r, w = make(M, F, dtype, 4), make(M, F, dtype, 5, 2.0), 1.0 + 0.3 * make(1, F, "f32", 6)[0]
    x[1] *= 1e-3
    x[M // 2] = 0
    r[M // 2] = 0
    s = state(F + 1)
    for p, res in ((0.0, None), (0.5, r)):
        y, h, rstd = ref.norm(x, w, EPS, res, p, s.tolist())
        off_y, off_h, off_rstd = ref.norm_bounds(x, w, y, h, rstd, t, res, p)
        buf, q = ref.guarded((M, F), torch.float8_e4m3fn, 3.0, shift=1)
        Q, scale, S, R = B.fastgl_norm_fwd_e4m3(x.cuda(), w.cuda(), EPS, residual=None if res is None else res.cuda(), rng=s, p=p, Q=q)
        want = (y.abs().amax(1) / 448).clamp_min(2.0 ** -126)
        assert_within(scale, want, off_y.amax(1) / 448 + 3 * ref.U32 * want, (F, p, "scale"))
        assert_within(R, rstd, off_rstd, (F, p, "rstd"))
        # half a step of e4m3 (normal, then subnormal) of y / scale, which carries y's error, the reciprocal's and the product's
        sc = scale.double().cpu()[:, None]
        bound = off_y + 4 * ref.U32 * y.abs() + (2.0 ** -4 * (y.abs() + off_y) * (1 + 4 * ref.U32) + sc * 2.0 ** -10)
        assert_within(Q.float().double().cpu() * sc, y, bound, (F, p, "q"))
        assert ref.bands_intact(buf, q, 3.0)
        zero = scale[M // 2].item() == 2.0 ** -126 and bool((Q[M // 2].float() == 0).all())
        assert zero
        # the table gathers back
        ids = torch.tensor([M - 1, 0, 0, M // 2, -1, M, 1], dtype=torch.int64, device="cuda")
        for d in ("f32", "bf16"):
            gb, go = ref.guarded((7, F), ref.DTYPES[d], SENTINEL, shift=1)
            B.fastgl_gather_rows_e4m3(Q.contiguous(), scale, ids, d, out=go)
            good = torch.tensor([0, 1, 2, 3, 6], device="cuda")
            exact = (Q.float()[ids[good]] * scale[ids[good]][:, None]).to(ref.DTYPES[d])     # one product, one rounding
            assert torch.equal(go[good], exact) and bool(torch.isnan(go[4:6]).all())
            assert ref.bands_intact(gb, go, SENTINEL)


def test_norm_rows_do_not_touch_each_other():
    x = make(50, 300, "f32", 7)
    w = torch.ones(300).cuda()
    clean, _, r0 = B.fastgl_norm_fwd(x.cuda(), w, EPS)
    x[3, 5], x[9, 299], x[20] = float("nan"), float("inf"), 0.0
    y, _, r1 = B.fastgl_norm_fwd(x.cuda(), w, EPS)
    Q, scale, _, _ = B.fastgl_norm_fwd_e4m3(x.cuda(), w, EPS)
    others = [i for i in range(50) if i not in (3, 9, 20)]
    assert torch.equal(y[others], clean[others]) and torch.equal(r1[others], r0[others])
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[9, 299])) and bool((y[9, :299] == 0).all())
    assert bool((y[20] == 0).all()) and abs(r1[20].item() * EPS ** 0.5 - 1) < 1e-6
    assert bool(torch.isnan(Q[3].float()).all()) and bool(torch.isfinite(scale[others]).all())


# --------------------------------------------------------------------------------- backward
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", WIDTHS)
def test_norm_backward(F, dtype):
    t = ref.DTYPES[dtype]
    for M, p, with_ds in ((1, 0.0, False), (rows_for(F), 0.3, True), (3 * rows_for(F), 0.0, True)):
        S, dY, dS = make(M, F, dtype, 1, 2.0), make(M, F, dtype, 2), make(M, F, dtype, 3)
        w = 1.0 + 0.3 * make(1, F, "f32", 4)[0]
        s = state(F)
        rstd = (1.0 / torch.sqrt(S.double().square().mean(1) + EPS)).float()
        dx, d, dw = ref.norm_grad(S, w, rstd, dY, dS if with_ds else None, p, s.tolist())
        n, tt = (S.double() * rstd.double()[:, None]).abs(), (dY.double() * w.double()).abs()
        mean, dot = (tt * n).mean(1, keepdim=True), (tt * n).mean(1, keepdim=True)
        off = ref.U32 * (rstd.double()[:, None] * (4 * tt + n * (5 * dot + (ref.chain(F) + 4) * mean)) + 2 * d.abs()
                         + (dS.double().abs() if with_ds else 0.0)) * 1.01
        k = ref.drop_scale(p) if p else 1.0
        bufs = [ref.guarded((M, F), t, SENTINEL, shift=1), ref.guarded((M, F), t, SENTINEL, shift=3), ref.guarded((F,), torch.float32, SENTINEL, shift=1)]
        gx, gr, gw = B.fastgl_norm_bwd(ref.shifted(S), ref.shifted(w), rstd.cuda(), ref.shifted(dY, 3), dS=ref.shifted(dS) if with_ds else None, rng=s,
                                       p=p, dX=bufs[0][1], dR=bufs[1][1], dw=bufs[2][1])
        assert_within(gr, d, off + ref.HALF[t] * (d.abs() + off), (F, M, "dR"))
        kept = ref.keep(M, F, p, s.tolist()) if p else torch.ones(M, F, dtype=torch.bool)
        assert_within(gx, dx, (k * off + ref.U32 * dx.abs() + ref.HALF[t] * (dx.abs() + k * off)) * kept * 1.01, (F, M, "dX"))
        lane_rows = min(M, 8 + M // 256)
        assert_within(gw, dw, ref.U32 * (lane_rows + 10) * (dY.double().abs() * n).sum(0), (F, M, "dw"))
        for buf, inner in bufs:
            assert ref.bands_intact(buf, inner, SENTINEL)
        again = B.fastgl_norm_bwd(S.cuda(), w.cuda(), rstd.cuda(), dY.cuda(), dS=dS.cuda() if with_ds else None, rng=s, p=p)
        assert torch.equal(again[0], gx) and torch.equal(again[1], gr) and torch.equal(again[2], gw)      # bit for bit
        only = B.fastgl_norm_bwd(S.cuda(), w.cuda(), rstd.cuda(), dY.cuda(), dS=dS.cuda() if with_ds else None, rng=s, p=p, want=("dw",))
        assert only[0] is None and only[1] is None and torch.equal(only[2], gw)


def test_norm_backward_without_rows_and_with_many():
    w = torch.ones(40).cuda()
    dx, dr, dw = B.fastgl_norm_bwd(torch.empty(0, 40).cuda(), w, torch.empty(0).cuda(), torch.empty(0, 40).cuda())
    assert dx.shape == (0, 40) and bool((dw == 0).all())
    M = 300_000
    S, dY = make(M, 40, "bf16", 1), make(M, 40, "bf16", 2)
    rstd = (1.0 / torch.sqrt(S.double().square().mean(1) + EPS)).float()
    _, _, dw = B.fastgl_norm_bwd(S.cuda(), w, rstd.cuda(), dY.cuda(), want=("dw",))
    n = S.double() * rstd.double()[:, None]
    assert_within(dw, (dY.double() * n).sum(0), ref.U32 * (8 + M // 256 + 10) * (dY.double() * n).abs().sum(0), "dw")


# --------------------------------------------------------------------------------- how it is called
def test_refusals_of_the_binding():
    x, w = torch.ones(4, 8).cuda(), torch.ones(8).cuda()
    for bad in (dict(X=x.cpu()), dict(X=x.double()), dict(X=torch.ones(8, 4).cuda().t()), dict(weight=w.cpu()), dict(weight=w.bfloat16()),
                dict(residual=x.bfloat16()), dict(rng=torch.zeros(2, device="cuda"), p=0.5)):
        with pytest.raises(TypeError):
            B.fastgl_norm_fwd(**{**dict(X=x, weight=w, eps=EPS), **bad})
    for bad in (dict(weight=w[:7].contiguous()), dict(residual=torch.ones(4, 7).cuda()), dict(Y=torch.ones(4, 7).cuda()), dict(X=x[0]),
                dict(rng=torch.zeros(3, dtype=torch.int64, device="cuda"), p=0.5)):
        with pytest.raises(ValueError):
            B.fastgl_norm_fwd(**{**dict(X=x, weight=w, eps=EPS), **bad})
    for bad in (dict(p=0.5), dict(p=2.0), dict(eps=-1.0)):
        with pytest.raises(B.FastglError):
            B.fastgl_norm_fwd(**{**dict(X=x, weight=w, eps=EPS), **bad})
    with pytest.raises(ValueError):
        B.fastgl_norm_bwd(x, w, torch.ones(3).cuda(), x)
    with pytest.raises(TypeError):
        B.fastgl_norm_bwd(x, w, torch.ones(4).cuda(), None)
    with pytest.raises(B.FastglError):
        B.fastgl_norm_bwd(x, w, torch.ones(4).cuda(), x, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    q = torch.zeros(4, 8, device="cuda").to(torch.float8_e4m3fn)
    with pytest.raises(TypeError):
        B.fastgl_gather_rows_e4m3(x, torch.ones(4).cuda(), torch.zeros(2, dtype=torch.int64).cuda(), "f32")
    with pytest.raises(ValueError):
        B.fastgl_gather_rows_e4m3(q, torch.ones(3).cuda(), torch.zeros(2, dtype=torch.int64).cuda(), "f32")
    with pytest.raises(TypeError):
        B.fastgl_gather_rows_e4m3(q, torch.ones(4).cuda(), torch.zeros(2, dtype=torch.int32).cuda(), "f32")


def test_replays_of_a_graph_take_the_offset_they_find():
    x, r, w, s = make(200, 100, "bf16", 1).cuda(), make(200, 100, "bf16", 2).cuda(), torch.ones(100).cuda(), state()
    dy = make(200, 100, "bf16", 3).cuda()

    def step():
        y, h, rstd = B.fastgl_norm_fwd(x, w, EPS, residual=r, rng=s, p=0.4)
        return (y, h, rstd, *B.fastgl_norm_bwd(h, w, rstd, dy, rng=s, p=0.4), B.fastgl_dropout(x, s, 0.4))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    seen = []
    for k in range(4):
        s[1] += 1
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b), k
        seen.append(out[-1].clone())
    assert not torch.equal(seen[0], seen[1])


# --------------------------------------------------------------------------------- e4m3: the quotient
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", [8, 64, 128, 256, 1024, 2048, 8192, 16_384])
def test_e4m3_is_the_rounded_quotient(F, dtype):
    """Rows of ones have rstd = 1 where eps = 0 and F is a power of two, so that Y is the weights: any values, here those next to
    the middle of two e4m3 values times the scale.  Q is then the float32 quotient, rounded, bit for bit."""
    rng = np.random.default_rng(F)
    x = torch.ones(3, F, dtype=ref.DTYPES[dtype], device="cuda")
    middles = np.array([(1 + (2 * i + 1) / 16) * 2.0 ** e for e in range(-6, 9) for i in range(8)] + [(i + 0.5) * 2.0 ** -9 for i in range(8)])
    middles = middles[middles < 448]
    for k in range(24):
        most = np.float32(rng.uniform(1, 2) * 2.0 ** rng.integers(-118, 120) if k % 3 else rng.uniform(0.5, 8))
        scale = max(most / np.float32(448), np.float32(2.0 ** -126))
        y = (rng.choice(middles, F) * scale).astype(np.float32)
        for _ in range(2):                                          # up to two values away from it
            y = np.choose(rng.integers(0, 3, F), [y, np.nextafter(y, np.float32(0)), np.nextafter(y, np.float32(np.inf))])
        y = np.minimum(y, most) * rng.choice([-1, 1], F).astype(np.float32)
        y[rng.integers(F)] = most
        Q, got_scale, _, rstd = B.fastgl_norm_fwd_e4m3(x, torch.from_numpy(y).cuda(), 0.0)
        assert bool((rstd == 1).all()) and bool((got_scale.cpu() == float(scale)).all()), k
        want = torch.from_numpy(y / scale).to(torch.float8_e4m3fn).view(torch.uint8)
        assert all(torch.equal(row, want) for row in Q.view(torch.uint8).cpu()), (k, most, scale)


def test_e4m3_of_weights_that_are_not_finite():
    """An infinite weight makes the scale infinite: every finite value over it is 0, itself NaN."""
    for F in (64, 1024, 16_384):
        w = torch.linspace(0.5, 1.5, F)
        w[3], w[F - 1] = float("inf"), float("nan")
        Q, scale, _, _ = B.fastgl_norm_fwd_e4m3(torch.ones(2, F, device="cuda"), w.cuda(), 0.0)
        q = Q.float().cpu()
        assert bool(torch.isinf(scale).all()) and bool(torch.isnan(q[:, [3, F - 1]]).all())
        q[:, [3, F - 1]] = 0
        assert bool((q == 0).all())


def test_gradients_are_tensors_of_their_own():
    """Also without dropout, where dX and dR are the same values: a change of one leaves the other as it is."""
    S, dY, w = make(50, 72, "f32", 1).cuda(), make(50, 72, "f32", 2).cuda(), torch.ones(72).cuda()
    rstd = (1.0 / torch.sqrt(S.double().square().mean(1) + EPS)).float()
    for p in (0.0, 0.3):
        dX, dR, dw = B.fastgl_norm_bwd(S, w, rstd, dY, rng=state(), p=p)
        kept = dR.clone()
        assert p > 0 or torch.equal(dX, dR)
        dX.zero_()
        assert torch.equal(dR, kept)
        for want, i in (("dX", 0), ("dR", 1)):                     # one of them alone
            alone = B.fastgl_norm_bwd(S, w, rstd, dY, rng=state(), p=p, want=(want,))
            assert [v is not None for v in alone] == [i == 0, i == 1, False]
            assert torch.equal(alone[1], kept) if i else p > 0 or torch.equal(alone[0], kept)
