"""The loss's entry points without a GPU: the coarse backward pass's refusals, workspaces over the whole range of sizes."""
import ctypes

from paper_2409_14939_amd import binding as B

FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001)
INVALID, UNSUPPORTED, WORKSPACE = B.FASTGL_ERR_INVALID_ARG, B.FASTGL_ERR_UNSUPPORTED, B.FASTGL_ERR_WORKSPACE


def test_coarse_calls_are_checked_alike():
    def coarse(dt=1, H=FAKE, M=64, K=8, N=512, dloss=FAKE, dW=FAKE, ws=FAKE, wsb=1 << 50):
        return B.lib().fastgl_loss_bwd_coarse(dt, H, FAKE, None, FAKE, FAKE, dloss, M, K, N, FAKE, dW, None, ws, wsb, None)
    for kw, status in ((dict(dt=2), INVALID), (dict(M=-1), INVALID), (dict(N=2 ** 21 + 1), UNSUPPORTED), (dict(H=ODD), INVALID), (dict(dloss=None), INVALID),
                       (dict(dW=ODD), INVALID), (dict(ws=None), INVALID), (dict(wsb=64), WORKSPACE)):
        assert coarse(**kw) == status
    size = B.fastgl_loss_bwd_workspace_bytes
    for M, K, N in ((4096, 128, 4096), (8192, 512, 16_384)):
        assert size("bf16", M, K, N) > 2 * 2 * M * N and size("bf16", M, K, N, coarse=True) > 2 * M * N      # two pieces of dZ, one
        assert size("f32", M, K, N, coarse=True) == size("f32", M, K, N)
    assert coarse(M=4096, K=128, N=4096, wsb=size("bf16", 4096, 128, 4096, True, coarse=True) - 1) == WORKSPACE


def test_no_workspace_grows_with_rows_times_classes():
    """H and W packed, a piece of statistics (8 bytes for 64 classes of a row at most) or of dZ, sums of rows; over the whole range of sizes."""
    for dt in ("f32", "bf16"):
        for M in (1, 300, 8192, 32_768, 10 ** 6, 2 ** 20, 2 ** 22, 2 ** 26, 2 ** 31 - 1 - 1024):
            for N in (1, 47, 65_536, 10 ** 6, 2 ** 21):
                for K in (0, 1, 256, 512):
                    if M * K > 2 ** 38:
                        continue
                    for aligned in (False, True):
                        size = B.fastgl_loss_fwd_workspace_bytes(dt, M, K, N, aligned)
                        assert size <= 6 * M * (K + 8) + max(1 << 30, 6 * K * 512) + max(1 << 30, 8 * M * 4) + 12 * M + 4096, (dt, M, K, N, size)


def test_dz_has_no_more_columns_than_it_needs():
    """Where all classes are one piece: a multiple of 32 of them; H packed, sums of dH, dW and db beside it."""
    for dt, planes in (("f32", 3), ("bf16", 2)):
        for M in (70_000, 2 ** 21, 2 ** 21 + 1):
            for K, N in ((8, 2), (8, 47), (64, 65), (300, 200)):
                rows, cols = M + 256, (N + 31) // 32 * 32
                if 2 * planes * rows * cols > 1 << 30:
                    continue
                size = B.fastgl_loss_bwd_workspace_bytes(dt, M, K, N, True)
                assert size < 2 * planes * cols * (rows + 100) + 6 * M * (K + 8) + 6 * K * cols + 3 * 4 * M * K + 64 * 4 * K * N + M * cols // 4 + (1 << 20), (dt, M, K, N)
