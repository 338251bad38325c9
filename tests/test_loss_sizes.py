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
