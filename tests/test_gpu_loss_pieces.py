"""The loss's forward pass with the classes in several pieces, and launches of very many tiles: some rows against the 64-bit form."""
import pytest
import torch

from loss_ref import Loss
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu


def check_rows(H, W, b, label, loss, lse, rows):
    ref = Loss(H[rows], W, b, label[rows])
    for got, name in ((loss[rows], "loss"), (lse[rows], "lse")):
        want, off = getattr(ref, name), getattr(ref, "off_" + name)
        same = (got.double() == want)
        assert bool((off < 1e-2 * want[torch.isfinite(want)].abs().max()).all())
        assert bool((same | ((got.double() - want).abs() <= off + 2.0 ** -24 * (want.abs() + off))).all()), name


# more than one piece of statistics from 2^33 rows x classes on; classes that are no multiple of 8 are packed, piece by piece
@pytest.mark.parametrize("dtype,M,K,N", [("bf16", 300_000, 16, 40_000), ("bf16", 300_001, 9, 40_001), ("f32", 250_000, 8, 40_000), ("bf16", 1 << 22, 8, 65_536)])
def test_statistics_of_several_pieces(dtype, M, K, N):
    g = torch.Generator(device="cuda").manual_seed(4)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    H, W, b = make(M, K).to(t), (2.0 * make(K, N) / K ** 0.5).to(t), 0.5 * make(N)
    label = torch.randint(-1, N, (M,), generator=g, device="cuda")
    need = B.fastgl_loss_fwd_workspace_bytes(dtype, M, K, N, True)
    assert need < (3 << 30) and M * N > 1 << 33
    ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    loss, lse = B.fastgl_loss_fwd(H, W, b, label, workspace=ws[:need])
    assert bool((ws[need:] == 0xA5).all())
    rows = torch.cat((torch.arange(60), torch.arange(M // 2, M // 2 + 60), torch.arange(M - 60, M))).cuda()
    check_rows(H, W, b, label, loss, lse, rows)
    assert bool(torch.isfinite(loss).all()) and not bool(loss[label < 0].any())
    ws[:need] = 0xFF
    again = B.fastgl_loss_fwd(H, W, b, label, workspace=ws[:need])
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
    # classes that are ruled out: all of the first piece, all of the last, all of them
    label[label >= 0] = N // 2
    b[:N // 2 - 100] = -float("inf")
    loss, lse = B.fastgl_loss_fwd(H, W, b, label, workspace=ws[:need])
    check_rows(H, W, b, label, loss, lse, rows)
    b[N // 2 + 100:] = torch.finfo(torch.float32).min
    loss, lse = B.fastgl_loss_fwd(H, W, b, label, workspace=ws[:need])
    check_rows(H, W[:, N // 2 - 100:N // 2 + 100], b[N // 2 - 100:N // 2 + 100], torch.where(label < 0, -1, 100), loss, lse, rows)
    b[:] = -float("inf")
    assert bool((B.fastgl_loss_fwd(H, W, b, label)[1] == -float("inf")).all())


def test_more_rows_than_tiles_of_512_threads_have():
    """A launch has less than 2^32 threads: 2^30 rows are 2^23 tiles of 256."""
    M, N = (1 << 30) + 5, 2
    H = torch.zeros(M, 1, device="cuda", dtype=torch.bfloat16)
    label = torch.full((M,), -1, device="cuda", dtype=torch.int64)
    g = torch.Generator(device="cuda").manual_seed(6)
    parts = [slice(at, at + 1000) for at in (0, M // 2, M - 1000)]
    for part in parts:
        H[part] = torch.randn(1000, 1, generator=g, device="cuda").bfloat16()
        label[part] = torch.randint(-1, N, (1000,), generator=g, device="cuda")
    W, b = torch.randn(1, N, generator=g, device="cuda").bfloat16(), torch.randn(N, generator=g, device="cuda")
    loss, lse = B.fastgl_loss_fwd(H, W, b, label)
    rows = torch.cat([torch.arange(p.start, p.stop) for p in parts]).cuda()
    check_rows(H, W, b, label, loss, lse, rows)
    between = slice(1000, M // 2)
    assert bool((lse[between] == lse[1000]).all()) and not bool(loss[between].any())


@pytest.mark.parametrize("coarse", [False, True])
def test_a_captured_step_of_several_pieces(coarse):
    """Statistics carried from piece to piece, dZ and dH by pieces: replays on other inputs, with a workspace that holds anything."""
    M, K, N = 300_000, 8, 40_000
    g = torch.Generator(device="cuda").manual_seed(5)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")
    sets = [[make(M, K).bfloat16(), make(K, N).bfloat16(), make(N), torch.randint(-1, N, (M,), generator=g, device="cuda"), make(M)] for _ in range(2)]
    need = max(B.fastgl_loss_fwd_workspace_bytes("bf16", M, K, N, True), B.fastgl_loss_bwd_workspace_bytes("bf16", M, K, N, True, coarse=coarse))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step(H, W, b, label, dloss):
        loss, lse = B.fastgl_loss_fwd(H, W, b, label, workspace=ws)
        return [loss, lse, *B.fastgl_loss_bwd(H, W, b, label, lse, dloss, workspace=ws, coarse=coarse)]
    eager = [[x.clone() for x in step(*s)] for s in sets]
    held = [x.clone() for x in sets[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step(*held)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            got = step(*held)
    torch.cuda.current_stream().wait_stream(side)
    for n in (0, 1, 0):
        for to, x in zip(held, sets[n]):
            to.copy_(x)
        for t in got:
            t.zero_()
        ws.random_(0, 255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager[n])), n
