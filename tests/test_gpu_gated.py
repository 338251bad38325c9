"""Gated feed-forward update on the GPU against its plain 64-bit form (tests/gated_ref.py)."""
import pytest
import torch

import gated_ref as ref
import rows_ref
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
SENTINEL = -776.0
U32 = ref.U32
# rows: below, at and beyond the line of the few-rows kernel and of a tile; widths: multiples of 8 and not, below and beyond a step of 64
SHAPES = [(1, 1, 1), (1, 256, 1024), (2, 5, 9), (3, 64, 64), (7, 100, 47), (16, 130, 200), (17, 8, 8), (17, 1, 1), (33, 7, 5), (48, 72, 80), (49, 33, 31), (64, 64, 64),
          (65, 72, 40), (100, 63, 65), (127, 128, 130), (129, 200, 48), (255, 256, 256), (257, 100, 136), (300, 602, 91), (513, 48, 700),
          (1000, 256, 683), (2100, 520, 264)]


def make(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(rows_ref.DTYPES[dtype])


def inputs(M, K, N, dtype, seed=0):
    x = make((M, K), dtype, seed + 1)
    wg, wu = make((K, N), dtype, seed + 2, K ** -0.5), make((K, N), dtype, seed + 3, K ** -0.5)
    bg, bu = make((N,), "f32", seed + 4, 0.3), make((N,), "f32", seed + 5, 0.3)
    return x, wg, wu, bg, bu


def within(got, want, bound, what):
    got, want = got.double().cpu(), want.double()
    assert got.shape == want.shape, what
    over = (got - want).abs() - bound
    assert bool(torch.isfinite(got).all()) and bool((over <= 0).all()), (what, over.max().item(), (got - want).abs().max().item(), want.abs().max().item())


def product_bound(a, b, terms, dtype):
    """Largest error of a @ b: a rounding per accumulated term of the sum's size (six piece products each for float32, their
    dropped rest 2^-23), the sum's size at most that of the magnitudes."""
    size = a.double().abs() @ b.double().abs()
    return size * (U32 * (terms + 2) * (1.2 if dtype == "bf16" else 1.3) + (2.0 ** -23 if dtype == "f32" else 0.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_forward(M, K, N, dtype):
    t = rows_ref.DTYPES[dtype]
    x, wg, wu, bg, bu = inputs(M, K, N, dtype)
    for n, name in enumerate(ref.ACTS):
        biases = ((bg, bu), (None, None), (bg, None), (None, bu))[n]
        p, g, u = ref.forward(x, wg, wu, *biases, name)
        extra = [0.0 if b is None else 2 * U32 * b.double().abs() for b in biases]
        off_g = product_bound(x, wg, K, dtype) + extra[0] + 2 * U32 * g.abs()
        off_u = product_bound(x, wu, K, dtype) + extra[1] + 2 * U32 * u.abs()
        a, _ = ref.act(name, g)
        # |act'| <= 1.13 (gelu), 1.1 (silu), 1, 1/4
        off_a = 1.13 * off_g + ref.off_act(name, g)[0]
        off_p = off_a * (u.abs() + off_u) + a.abs() * off_u + U32 * p.abs()
        shift = n % 3                                             # starts that are multiples of 16 bytes and not
        bufs = [rows_ref.guarded((M, N), t, SENTINEL, shift=shift) for _ in range(3)]
        args = [rows_ref.shifted(v, 8 if shift == 0 else shift) if v is not None else None for v in (x, wg, wu, *biases)]
        P, G, U = B.fastgl_gated_fwd(*args, name, P=bufs[0][1], G=bufs[1][1], U=bufs[2][1])
        within(G, g, off_g + ref.HALF[t] * (g.abs() + off_g), (name, "G"))
        within(U, u, off_u + ref.HALF[t] * (u.abs() + off_u), (name, "U"))
        within(P, p, off_p + ref.HALF[t] * (p.abs() + off_p) + 1e-38, (name, "P"))
        for buf, inner in bufs:
            assert rows_ref.bands_intact(buf, inner, SENTINEL)
        P2, G2, U2 = B.fastgl_gated_fwd(*args, name, want_GU=False)
        assert G2 is None and U2 is None and torch.equal(P2, P)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_backward(M, K, N, dtype):
    t = rows_ref.DTYPES[dtype]
    x, wg, wu, _, _ = inputs(M, K, N, dtype, 10)
    g, u, dp = make((M, N), dtype, 21, 1.5), make((M, N), dtype, 22), make((M, N), dtype, 23)
    for n, name in enumerate(ref.ACTS):
        dx, dwg, dwu, dbg, dbu, dg, du = ref.backward(x, wg, wu, g, u, dp, name)
        oa, oda = ref.off_act(name, g)
        pu = (dp.double() * u.double()).abs()
        off_dg, off_du = pu * oda + 3 * U32 * dg.abs(), dp.double().abs() * oa + 2 * U32 * du.abs()
        half = 0.0 if dtype == "f32" else ref.HALF[t]             # dG and dU are rounded on their way to the products
        in_g, in_u = off_dg + half * (dg.abs() + off_dg), off_du + half * (du.abs() + off_du)
        off_x = in_g @ wg.double().abs().T + in_u @ wu.double().abs().T + product_bound(dg, wg.T, 2 * N, dtype) + product_bound(du, wu.T, 2 * N, dtype)
        xa = x.double().abs().T
        off_wg, off_wu = xa @ in_g + product_bound(x.T, dg, M, dtype), xa @ in_u + product_bound(x.T, du, M, dtype)
        shift = n % 3
        shapes = ((M, K), (K, N), (K, N), (N,), (N,))
        bufs = [rows_ref.guarded(s, t if i < 3 else torch.float32, SENTINEL, shift=shift) for i, s in enumerate(shapes)]
        args = [rows_ref.shifted(v, 8 if shift == 0 else shift) for v in (x, wg, wu, g, u, dp)]
        out = B.fastgl_gated_bwd(*args, name, dX=bufs[0][1], dWg=bufs[1][1], dWu=bufs[2][1], dbg=bufs[3][1], dbu=bufs[4][1])
        for got, want, off, what in ((out[0], dx, off_x, "dX"), (out[1], dwg, off_wg, "dWg"), (out[2], dwu, off_wu, "dWu")):
            within(got, want, off * 1.01 + ref.HALF[t] * (want.abs() + off) + 1e-38, (name, what))
        within(out[3], dbg, off_dg.sum(0) + U32 * (M + 20) * dg.abs().sum(0) + 1e-38, (name, "dbg"))
        within(out[4], dbu, off_du.sum(0) + U32 * (M + 20) * du.abs().sum(0) + 1e-38, (name, "dbu"))
        for buf, inner in bufs:
            assert rows_ref.bands_intact(buf, inner, SENTINEL)
        for want in (("dX",), ("dWu",), ("dbg",), ("dWg", "dbu")):    # parts: the same bits, the others None
            part = B.fastgl_gated_bwd(*args, name, want=want)
            for i, key in enumerate(("dX", "dWg", "dWu", "dbg", "dbu")):
                assert (part[i] is not None and torch.equal(part[i], out[i])) if key in want else part[i] is None


@pytest.mark.parametrize("dtype,M,K,N", [("bf16", 20_000, 256, 200), ("bf16", 5000, 1024, 1032), ("f32", 9000, 130, 260), ("bf16", 70_001, 64, 24)])
def test_many_tiles_and_slabs(dtype, M, K, N):
    """The large tiles, several slabs, partial tiles on every side; the same bits again."""
    t = rows_ref.DTYPES[dtype]
    x, wg, wu, bg, bu = (v.cuda() for v in inputs(M, K, N, dtype, 30))
    P, G, U = B.fastgl_gated_fwd(x, wg, wu, bg, bu, "silu")
    dp = make((M, N), dtype, 33).cuda()
    out = B.fastgl_gated_bwd(x, wg, wu, G, U, dp, "silu")
    again = B.fastgl_gated_bwd(x, wg, wu, G, U, dp, "silu")
    assert all(torch.equal(a, b) for a, b in zip(out, again))
    xd, wgd, wud = x.double(), wg.double(), wu.double()
    g = xd @ wgd + bg.double()
    bound = (xd.abs() @ wgd.abs()) * U32 * (K + 4) * 1.3 + (xd.abs() @ wgd.abs()) * 2.0 ** -23
    assert bool(((G.double() - g).abs() <= bound + ref.HALF[t] * (g.abs() + bound) + 4 * U32).all())
    dx, dwg, dwu, dbg, dbu, dg, du = ref.backward(x, wg, wu, G, U, dp, "silu")
    half = 2.0 ** -22 if dtype == "f32" else ref.HALF[t] * 1.01
    for got, want, size, terms in ((out[0], dx, dg.abs() @ wgd.abs().T + du.abs() @ wud.abs().T, 4 * N), (out[1], dwg, xd.abs().T @ dg.abs(), M),
                                   (out[2], dwu, xd.abs().T @ du.abs(), M)):
        off = size * (half + U32 * 1.3 * (terms + 4) + 2.0 ** -20)
        assert bool(((got.double() - want).abs() <= off + ref.HALF[t] * (want.abs() + off)).all())
    for got, want, size in ((out[3], dbg, dg.abs().sum(0)), (out[4], dbu, du.abs().sum(0))):
        assert bool(((got.double() - want).abs() <= size * 2.0 ** -18).all())


def test_what_is_not_finite_stays_in_its_row_and_column():
    for dtype in ("f32", "bf16"):
        for M in (9, 300, 1100):
            x, wg, wu, bg, bu = (v.cuda() for v in inputs(M, 72, 88, dtype, 40))
            clean = B.fastgl_gated_fwd(x, wg, wu, bg, bu, "silu")
            bad = x.clone()
            bad[4, 71], bad[M - 1, 0] = float("nan"), float("inf")
            w = wu.clone()
            w[3, 87] = float("nan")
            P, G, U = B.fastgl_gated_fwd(bad, wg, w, bg, bu, "silu")
            rows = [i for i in range(M) if i not in (4, M - 1)]
            assert bool(torch.isnan(G[4]).all()) and not bool(torch.isfinite(G[M - 1]).any()) and bool(torch.isnan(U[:, 87]).all())
            assert torch.equal(G[rows], clean[1][rows]) and torch.equal(U[rows][:, :87], clean[2][rows][:, :87])
            assert torch.equal(P[rows][:, :87], clean[0][rows][:, :87])
            dp = make((M, 88), dtype, 44).cuda()
            out0 = B.fastgl_gated_bwd(x, wg, wu, clean[1], clean[2], dp, "silu")
            dp[5, 87] = float("nan")
            out1 = B.fastgl_gated_bwd(x, wg, wu, clean[1], clean[2], dp, "silu")
            rows = [i for i in range(M) if i != 5]
            assert torch.equal(out0[0][rows], out1[0][rows]) and bool(torch.isnan(out1[0][5]).all())
            for a, b in zip(out0[1:], out1[1:]):
                assert torch.equal(a[..., :87], b[..., :87]) and bool(torch.isnan(b[..., 87]).all())


def test_sizes_of_zero():
    for dtype in ("f32", "bf16"):
        t = rows_ref.DTYPES[dtype]
        e = lambda *s: torch.ones(*s, device="cuda", dtype=t)  # noqa: E731
        bg, bu = torch.full((6,), 0.5).cuda(), torch.full((6,), 2.0).cuda()
        for M in (3, 40):                                         # no columns of X: the biases alone
            P, G, U = B.fastgl_gated_fwd(e(M, 0), e(0, 6), e(0, 6), bg, bu, "relu")
            assert bool((P == 1).all()) and bool((G == 0.5).all()) and bool((U == 2).all())
            dx, dwg, dwu, dbg, dbu = B.fastgl_gated_bwd(e(M, 0), e(0, 6), e(0, 6), G, U, e(M, 6), "relu")
            assert dx.shape == (M, 0) and dwg.shape == (0, 6) and bool((dbg == 2 * M).all()) and bool((dbu == 0.5 * M).all())
        P, G, U = B.fastgl_gated_fwd(e(0, 5), e(5, 6), e(5, 6), bg, bu)
        assert P.shape == (0, 6)
        dx, dwg, dwu, dbg, dbu = B.fastgl_gated_bwd(e(0, 5), e(5, 6), e(5, 6), G, U, e(0, 6))
        assert dx.shape == (0, 5) and all(bool((v == 0).all()) for v in (dwg, dwu, dbg, dbu))
        P, G, U = B.fastgl_gated_fwd(e(20, 5), e(5, 0), e(5, 0))
        assert P.shape == (20, 0)
        dx, dwg, _, _, _ = B.fastgl_gated_bwd(e(20, 5), e(5, 0), e(5, 0), G, U, e(20, 0))
        assert bool((dx == 0).all()) and dwg.shape == (5, 0)


def test_refusals_of_the_binding():
    x, w = torch.ones(20, 8).cuda(), torch.ones(8, 16).cuda()
    b = torch.ones(16).cuda()
    for bad in (dict(X=x.cpu()), dict(Wg=w.bfloat16()), dict(Wu=torch.ones(16, 8).cuda().t()), dict(bg=b.bfloat16())):
        with pytest.raises(TypeError):
            B.fastgl_gated_fwd(**{**dict(X=x, Wg=w, Wu=w, bg=b, bu=b), **bad})
    for bad in (dict(Wg=torch.ones(7, 16).cuda()), dict(Wu=torch.ones(8, 15).cuda()), dict(bg=torch.ones(8).cuda()), dict(P=torch.ones(20, 15).cuda())):
        with pytest.raises(ValueError):
            B.fastgl_gated_fwd(**{**dict(X=x, Wg=w, Wu=w, bg=b, bu=b), **bad})
    with pytest.raises(KeyError):
        B.fastgl_gated_fwd(x, w, w, act="tanh")
    with pytest.raises(B.FastglError):
        B.fastgl_gated_fwd(x.repeat(5, 1), w, w, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        B.fastgl_gated_bwd(x, w, w, torch.ones(20, 16).cuda(), torch.ones(20, 15).cuda(), torch.ones(20, 16).cuda())


def test_replays_of_a_graph():
    x, wg, wu, bg, bu = (v.cuda() for v in inputs(300, 100, 91, "f32", 50))
    dp = make((300, 91), "f32", 51).cuda()

    def step():
        out = B.fastgl_gated_fwd(x, wg, wu, bg, bu, "gelu")
        return (*out, *B.fastgl_gated_bwd(x, wg, wu, out[1], out[2], dp, "gelu"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        x.mul_(1.25)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b), k


def test_more_rows_than_blocks_of_columns_take():
    """Beyond 2^22 rows dG and dU lie in whole rows."""
    M, K, N = (1 << 22) + 33, 8, 40
    g = torch.Generator(device="cuda").manual_seed(1)
    x, G, U, dp = (torch.randn(M, n, generator=g, device="cuda", dtype=torch.float32).bfloat16() for n in (K, N, N, N))
    wg, wu = (torch.randn(K, N, generator=g, device="cuda", dtype=torch.float32).bfloat16() for _ in range(2))
    dx, dwg, dwu, dbg, dbu = B.fastgl_gated_bwd(x, wg, wu, G, U, dp, "silu")
    want = ref.backward(x, wg, wu, G, U, dp, "silu")
    dg, du = want[5], want[6]
    size = dg.abs() @ wg.double().abs().T + du.abs() @ wu.double().abs().T
    off = size * (2.0 ** -8 * 1.01 + U32 * 4 * N) + 1e-6
    assert bool(((dx.double() - want[0]).abs() <= off + 2.0 ** -8 * (want[0].abs() + off)).all())
    for got, exact, term in ((dwg, want[1], dg), (dwu, want[2], du)):
        # independent roundings of 2^-8 at most of each term, float32 sums of slabs of some 10^5 terms, one rounding of the result
        noise = (x.double().square().T @ term.square()).sqrt() * 2.0 ** -8
        assert bool(((got.double() - exact).abs() <= 6 * noise + 2.0 ** -8 * exact.abs() + (x.double().abs().T @ term.abs()) * 2.0 ** -20).all())
    for got, exact, term in ((dbg, want[3], dg), (dbu, want[4], du)):
        assert bool(((got.double() - exact).abs() <= term.abs().sum(0) * 2.0 ** -18).all())


# --------------------------------------------------------------------------------- the gate alone
def gate_points(dtype):
    """2^14 gates in -10 .. 10, dense below 0."""
    v = torch.cat([torch.linspace(-10, 0, 10_000), torch.linspace(0, 10, 6384)])
    return v.to(rows_ref.DTYPES[dtype])


def gate_bounds(name, dtype, g):
    """Relative error of act(g) before it is rounded to its type.  GELU: the tail 8.4 U32 (two roundings of t, which count three times at
    most in the polynomial, one of it and of the exponential, which the hardware gives within 2^-23, and the exponent), bf16 4e-5 of the
    fit; 1 - tail doubles the absolute share at most; the product.  SiLU, sigmoid: exponent, exponential, sum, reciprocal, product."""
    if name == "gelu":
        return 20 * U32 + (4e-5 + 2 * U32 * g.square() if dtype == "bf16" else 0.0) * torch.ones_like(g)
    return (0.0 if name == "relu" else 8 * U32 + 2 * U32 * g.abs()) * torch.ones_like(g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ref.ACTS)
def test_gates_keep_their_digits(name, dtype):
    """P without columns of X is act(bg) * 1, and the column sums of one row are dU = act(G), dG = act'(G): exact in relative terms, far below 0
    too."""
    t = rows_ref.DTYPES[dtype]
    g = gate_points(dtype)
    N, ones = g.numel(), torch.ones(g.numel()).cuda()
    gd = g.double()
    a, da = ref.act(name, gd)
    rel = gate_bounds(name, dtype, gd)
    e = lambda *s: torch.empty(*s, device="cuda", dtype=t)  # noqa: E731
    for M in (1, 300):                                              # the kernel of few rows, the tiles
        P, _, _ = B.fastgl_gated_fwd(e(M, 0), e(0, N), e(0, N), g.float().cuda(), ones, name)
        off = rel * a.abs()
        for row in (P[0], P[M - 1]):
            within(row, a, off + ref.HALF[t] * (a.abs() + off) + 1e-37, (name, M))
    one = torch.ones(1, N, device="cuda", dtype=t)
    _, _, _, dbg, dbu = B.fastgl_gated_bwd(one[:, :1].contiguous(), e(1, N), e(1, N), g.cuda().view(1, N), one, one, name, want=("dbg", "dbu"))
    within(dbu, a, rel * a.abs() + 2 * U32 * a.abs() + 1e-37, (name, "dbu"))
    if name == "gelu":
        cdf, pdf = 0.5 * torch.special.erfc(-gd / 2 ** 0.5), torch.exp(-0.5 * gd * gd) / (2 * torch.pi) ** 0.5
        off = rel * cdf + gd.abs() * pdf * (12 * U32 + (2 * U32 * gd.square() if dtype == "bf16" else 0.0)) + 3 * U32 * da.abs()
    elif name == "silu":
        s = torch.sigmoid(gd)
        off = rel * s * (1 + gd.abs()) + 4 * U32 * (s * (1 + gd.abs() * (1 - s))) + s * gd.abs() * (U32 + rel * s)
    else:
        off = rel * a.abs() * (1 + a.abs()) + 4 * U32 * a.abs() + U32 * a.abs()
    within(dbg, da, (off if name != "relu" else 0.0 * gd) + 1e-37, (name, "dbg"))


def test_gate_of_what_is_not_finite_and_far_out():
    inf = float("inf")
    for dtype in ("f32", "bf16"):
        t = rows_ref.DTYPES[dtype]
        g = torch.tensor([inf, 3e38, 1e20, 100.0, 0.0, -0.0, -100.0, -1e20, -3e38, -inf, float("nan")])
        N = g.numel()
        e = lambda *s: torch.empty(*s, device="cuda", dtype=t)  # noqa: E731
        for M in (2, 300):
            P, _, _ = B.fastgl_gated_fwd(e(M, 0), e(0, N), e(0, N), g.cuda(), torch.ones(N).cuda(), "gelu")
            p = P[M - 1].float().cpu()
            assert torch.equal(p[:4], g[:4].to(t).float()) and bool((p[4:9] == 0).all()) and bool(torch.isnan(p[9:]).all())


# --------------------------------------------------------------------------------- what dG and dU are rounded to
@pytest.mark.parametrize("M,K,N", [(1, 8, 16), (1, 256, 1024), (4, 16, 300), (16, 64, 1024), (17, 64, 1024), (30, 100, 300), (300, 32, 32), (300, 33, 32),
                                   (1030, 40, 72), (20_000, 256, 200)])
def test_terms_of_bf16_gradients(M, K, N):
    """One rule at every size.  With ReLU dG = dP U and dU = dP G are exact in float32, so that their roundings to bfloat16 are known: the plain call
    gives the products of those, the fine one those of the unrounded terms."""
    x, wg, wu, _, _ = inputs(M, K, N, "bf16", 60)
    g, u, dp = make((M, N), "bf16", 71), make((M, N), "bf16", 72), make((M, N), "bf16", 73)
    on = (g > 0).double()
    dg, du = dp.double() * u.double() * on, dp.double() * g.double() * on
    args = [v.cuda() for v in (x, wg, wu, g, u, dp)]
    for fine, half in ((False, 0.0), (True, 2.0 ** -17)):
        a, b = (v if fine else v.bfloat16().double() for v in (dg, du))
        out = B.fastgl_gated_bwd(*args, "relu", want=("dX", "dWg", "dWu"), fine=fine)
        xd, wgd, wud = x.double(), wg.double(), wu.double()
        for got, want, size, terms, what in ((out[0], a @ wgd.T + b @ wud.T, a.abs() @ wgd.abs().T + b.abs() @ wud.abs().T, 2 * N, "dX"),
                                             (out[1], xd.T @ a, xd.abs().T @ a.abs(), M, "dWg"), (out[2], xd.T @ b, xd.abs().T @ b.abs(), M, "dWu")):
            off = size * (half + U32 * 1.3 * (terms * (2 if fine else 1) + 4))
            within(got, want, off + 2.0 ** -8 * (want.abs() + off) + 1e-37, (fine, what))
    f32 = [v.float() for v in args]
    for p, q in zip(B.fastgl_gated_bwd(*f32, "relu"), B.fastgl_gated_bwd(*f32, "relu", fine=True)):
        assert torch.equal(p, q)
