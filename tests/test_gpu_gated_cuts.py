"""Every cut of the gated update's products - tile sizes, slabs, results past the caches, lanes a row of the kernel of few rows - on the GPU:
whole numbers by equality, so that a term that is left out or counted twice shows, and random ones against 64 bits there."""
import pytest
import torch

import gated_ref as ref
import rows_ref
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
U32 = ref.U32
# (M, K, N) and what the launch model takes for forward, dX, dW there: L, M, S the tile, p slabs, o results past the caches.
SHAPES_BF16 = [(34_534, 194, 81),      # L, L, S p
               (1552, 200, 2560),      # L o, S p, S p
               (8709, 1999, 198),      # L p, M, M p
               (18_291, 8, 71),        # M, S, S p
               (524, 16, 3392),        # M o, S p, S p
               (11, 1656, 4224),       # M p, S p, L
               (12, 632, 8),           # S p, S, S
               (56_828, 138, 8),       # S, L, S p
               (18_692, 141, 770),     # M, L p, M p
               (17_470, 154, 8),       # S, M, S p
               (9, 936, 4800),         # S p, M p, L
               (9, 1074, 3729),        # few rows, S p, L
               (2900, 137, 4178),      # M, S p, L p
               (9, 410, 4586),         # few rows, S p, M
               (8186, 8, 481),         # M, S p, M p
               (1106, 1461, 479), (54, 1096, 2686), (2492, 1471, 2596), (70_001, 64, 24), (115_000, 256, 1024), (16_384, 1024, 4096)]
SHAPES_F32 = [(17_719, 34, 193),       # L, S p, S p
              (40_729, 35, 96),        # L o, S, S p
              (17_433, 263, 68),       # L p, S, M p
              (17_250, 9, 83),         # M, S, S p
              (22_255, 9, 128),        # M o, S, S p
              (50, 1528, 1728),        # few rows, M p, M
              (50, 72, 9),             # few rows, S, S
              (39_388, 145, 9),        # S, L, S p
              (17_322, 136, 128),      # M o, L p, S p
              (18_948, 151, 8),        # S, M, S p
              (9, 1192, 757),          # few rows, M p, S
              (9, 920, 4352),          # few rows, M p, L
              (5131, 908, 65),         # S p, M, L p
              (9, 1326, 1480),         # few rows, S p, M
              (1327, 9, 455),          # S, S p, M p
              (64, 1528, 1728),        # S p, S p, M
              (64, 72, 9),             # S p, S, S
              (372, 1046, 4427),       # M p, S p, L
              (61, 300, 100), (33_388, 82, 2900), (70_001, 64, 24), (4000, 1024, 1500)]
# dG and dU lie in blocks of 32 columns from 1024 rows on.
LINES = [(1023, 40, 100), (1024, 40, 100), (1025, 33, 65)]
SHAPES = [("bf16", *s) for s in SHAPES_BF16 + LINES] + [("f32", *s) for s in SHAPES_F32 + LINES]
# Lanes a row of the kernel of few rows: 1, 2, 4 and 8 from 1, 3057, 6113 and 12225 columns on; rows of which it has 1, 2 or 4 a workgroup.
FEW = [(dtype, M, K, N) for dtype in ("f32", "bf16") for N in (2501, 3057, 4099, 6113, 7000, 12_225, 12_230) for M, K in ((1, 100), (2, 257), (3, 31), (8, 64))]
FEW += [("f32", M, 65, N) for M in (5, 47, 48) for N in (1000, 3060, 6120, 12_240)]


def pattern(g, terms, columns):
    """[terms, columns] of whole numbers whose sums down the columns are small, while part of the terms hardly ever sums to 0."""
    half = terms // 2
    a = torch.randint(1, 3, (half, columns), generator=g, device="cuda") * (2 * torch.randint(0, 2, (half, columns), generator=g, device="cuda") - 1)
    p = torch.cat([a, -a[torch.randperm(half, generator=g, device="cuda")], torch.ones(terms - 2 * half, columns, device="cuda", dtype=torch.int64)])
    p[torch.randint(0, terms, (1,), generator=g, device="cuda")] += 1
    return p


def pick(g, values, *shape):
    v = torch.tensor(values, device="cuda")
    return v[torch.randint(0, len(values), shape, generator=g, device="cuda")]


def equal(got, want, what):
    """`want` is exact; the result is its rounding."""
    assert torch.equal(got, want.to(got.dtype)), (what, (got.double() - want).abs().max().item())


def whole(dtype, M, K, N):
    g, t = torch.Generator(device="cuda").manual_seed(M + K + N), rows_ref.DTYPES[dtype]
    return g, lambda v: v.to(t).contiguous()


def forward_of_whole_numbers(dtype, M, K, N):
    g, cast = whole(dtype, M, K, N)
    x, wg, wu = cast(pick(g, [-1, 1, 2], M, 1).expand(M, K)), cast(pattern(g, K, N)), cast(pattern(g, K, N))
    bg, bu = pick(g, [-3, 2, 5], N).float(), pick(g, [-2, 1, 4], N).float()
    P, G, U = B.fastgl_gated_fwd(x, wg, wu, bg, bu, "relu")
    gd, ud = x.double() @ wg.double() + bg, x.double() @ wu.double() + bu
    equal(G, gd, "G")
    equal(U, ud, "U")
    equal(P, gd.clamp_min(0) * ud, "P")
    alone = B.fastgl_gated_fwd(x, wg, wu, bg, bu, "relu", want_GU=False)
    assert torch.equal(alone[0], P) and alone[1] is None


@pytest.mark.parametrize("dtype,M,K,N", SHAPES + FEW)
def test_forward_counts_every_term_once(dtype, M, K, N):
    forward_of_whole_numbers(dtype, M, K, N)


# The last: beyond 2^22 rows they lie in whole rows again.
@pytest.mark.parametrize("dtype,M,K,N", SHAPES + [("bf16", (1 << 22) + 33, 8, 40)])
def test_gradients_count_every_term_once(dtype, M, K, N):
    g, cast = whole(dtype, M, K, N)
    # dX: the terms are columns of G and U
    ones = cast(torch.ones(M, N, device="cuda"))
    wg, wu = cast(pattern(g, N, K).t()), cast(pattern(g, N, K).t())
    x, dp = cast(torch.ones(M, K, device="cuda")), cast(pick(g, [-1, 1, 2], M, 1).expand(M, N))
    for fine in (False, True) if dtype == "bf16" else (False,):
        dx, *_ = B.fastgl_gated_bwd(x, wg, wu, ones, ones, dp, "relu", want=("dX",), fine=fine)
        equal(dx, dp.double() @ (wg.double() + wu.double()).t(), ("dX", fine))
    # dWg, dWu, dbg, dbu: the terms are rows
    x, dp = cast(pick(g, [-1, 1, 2], 1, K).expand(M, K)), cast(pattern(g, M, N))
    G, U = cast(pick(g, [1, 2], 1, N).expand(M, N)), cast(pick(g, [-1, 1], 1, N).expand(M, N))
    dg, du = dp.double() * U.double(), dp.double() * G.double()
    for fine in (False, True) if dtype == "bf16" else (False,):
        _, dwg, dwu, dbg, dbu = B.fastgl_gated_bwd(x, wg, wu, G, U, dp, "relu", want=("dWg", "dWu", "dbg", "dbu"), fine=fine)
        equal(dwg, x.double().t() @ dg, ("dWg", fine))
        equal(dwu, x.double().t() @ du, ("dWu", fine))
        equal(dbg, dg.sum(0), "dbg")
        equal(dbu, du.sum(0), "dbu")


def inputs(dtype, M, K, N):
    g, t = torch.Generator(device="cuda").manual_seed(M + K), rows_ref.DTYPES[dtype]
    make = lambda scale, *s: (scale * torch.randn(*s, generator=g, device="cuda")).to(t)  # noqa: E731
    return make, make(1, M, K), make(K ** -0.5, K, N), make(K ** -0.5, K, N), make(0.3, N).float(), make(0.3, N).float()


def within(got, want, bound, what):
    over = (got.double() - want).abs() - bound
    assert bool((over <= 0).all()), (what, over.max().item())


def sum_bound(size, terms, dtype):
    """A rounding per term of the sum's size, and what six of nine piece products leave."""
    return size * (U32 * (terms + 4) * 1.3 + (2.0 ** -23 if dtype == "f32" else 0.0))


@pytest.mark.parametrize("dtype,M,K,N", SHAPES + FEW)
def test_forward_against_64_bits(dtype, M, K, N):
    t, name = rows_ref.DTYPES[dtype], ref.ACTS[(M + N) % 4]
    _, x, wg, wu, bg, bu = inputs(dtype, M, K, N)
    P, G, U = B.fastgl_gated_fwd(x, wg, wu, bg, bu, name)
    xd, wgd, wud = x.double(), wg.double(), wu.double()
    g, u = xd @ wgd + bg.double(), xd @ wud + bu.double()
    off_g = sum_bound(xd.abs() @ wgd.abs(), K, dtype) + 2 * U32 * (bg.double().abs() + g.abs())
    off_u = sum_bound(xd.abs() @ wud.abs(), K, dtype) + 2 * U32 * (bu.double().abs() + u.abs())
    a, _ = ref.act(name, g)
    off_a = 1.13 * off_g + ref.off_act(name, g)[0] + (1e-6 * g.abs() if dtype == "bf16" and name == "gelu" else 0.0)
    off_p = off_a * (u.abs() + off_u) + a.abs() * off_u + U32 * (a * u).abs()
    within(G, g, off_g + ref.HALF[t] * (g.abs() + off_g), "G")
    within(U, u, off_u + ref.HALF[t] * (u.abs() + off_u), "U")
    within(P, a * u, off_p + ref.HALF[t] * ((a * u).abs() + off_p) + 1e-37, "P")


@pytest.mark.parametrize("dtype,M,K,N", SHAPES)
def test_gradients_against_64_bits(dtype, M, K, N):
    t = rows_ref.DTYPES[dtype]
    make, x, wg, wu, _, _ = inputs(dtype, M, K, N)
    G, U, dp = make(1.5, M, N), make(1, M, N), make(1, M, N)
    out = B.fastgl_gated_bwd(x, wg, wu, G, U, dp, "silu")
    dx, dwg, dwu, dbg, dbu, dg, du = ref.backward(x, wg, wu, G, U, dp, "silu")
    oa, oda = ref.off_act("silu", G)
    # errors of the terms: formed in float32, then rounded where the type is bfloat16
    off_dg, off_du = (dp.double() * U.double()).abs() * oda + 3 * U32 * dg.abs(), dp.double().abs() * oa + 2 * U32 * du.abs()
    half = 0.0 if dtype == "f32" else ref.HALF[t]
    in_g, in_u = off_dg + half * (dg.abs() + off_dg), off_du + half * (du.abs() + off_du)
    xa, ga, ua = x.double().abs().t(), wg.double().abs().t(), wu.double().abs().t()
    for got, want, off, size, terms, what in ((out[0], dx, in_g @ ga + in_u @ ua, dg.abs() @ ga + du.abs() @ ua, 2 * N, "dX"),
                                              (out[1], dwg, xa @ in_g, xa @ dg.abs(), M, "dWg"), (out[2], dwu, xa @ in_u, xa @ du.abs(), M, "dWu")):
        off = (off + sum_bound(size, terms, dtype)) * 1.01
        within(got, want, off + ref.HALF[t] * (want.abs() + off) + 1e-37, what)
    within(out[3], dbg, off_dg.sum(0) + U32 * (M + 20) * dg.abs().sum(0) + 1e-37, "dbg")
    within(out[4], dbu, off_du.sum(0) + U32 * (M + 20) * du.abs().sum(0) + 1e-37, "dbu")
