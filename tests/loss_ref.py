"""Softmax cross entropy of class scores in 64 bits, and the largest errors of the kernels' float32 arithmetic from the same inputs."""
import torch

U32 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float64: 0.0}
LEAST = 2.0 ** -102                                       # weights below 2^-126 are 0: that times 2^24 terms at most


class Loss:
    """Scores, loss and lse, each with its bound: a score of K accumulated float32 terms is off by (K + 2) u of the sum of its terms' sizes
    and by 2^-23 of them where float32 products come from pieces; a weight by its score's error, lse's, and the rounding of its exponent."""

    def __init__(self, H, W, b, label):
        self.H, self.W, self.label, self.t = H.double(), W.double(), label, H.dtype
        f32 = H.dtype == torch.float32
        K, N = W.shape
        bias = torch.zeros(N, dtype=torch.float64) if b is None else b.double()
        self.z = self.H @ self.W + bias
        size = self.H.abs() @ self.W.abs() + torch.where(torch.isfinite(bias), bias.abs(), 0.0)
        # six accumulated piece products for float32, smallest first: a quarter more than the terms themselves
        self.off_z = size * (U32 * (K + 3) * 1.3 + (2.0 ** -23 if f32 else 0.0))
        self.lse = torch.logsumexp(self.z, 1)
        on = torch.where(torch.isfinite(self.z), self.z, 0.0)
        # weights: also the exponent's argument, and two units of the exponential itself
        self.rel = self.off_z + 2 * U32 * (2 + on.abs() + self.lse.abs()[:, None])
        p = torch.exp(self.z - self.lse[:, None])
        self.p = p
        # sums in float32 within a tile (at most 128 columns a lane pair: 64 terms), then over tiles
        self.off_lse = (p * self.rel).sum(1) + U32 * (64 + N / 64 + 16 + 2 * self.lse.abs())
        at = label.clamp(0, N - 1)[:, None]
        picked, off = self.z.gather(1, at)[:, 0], self.off_z.gather(1, at)[:, 0]
        self.on = label >= 0
        self.loss = torch.where(self.on, self.lse - picked, 0.0)
        self.off_loss = torch.where(self.on, self.off_lse + off + U32 * (self.lse.abs() + self.loss.abs()), 0.0)

    def backward(self, dloss):
        """dH, dW, db and off_ of each, for the kernels' own lse; products of dZ rounded to its operands' type."""
        N = self.W.shape[1]
        f32 = self.t == torch.float32
        g = torch.where(self.on, dloss.double(), 0.0)[:, None]
        hot = torch.zeros_like(self.p)
        hot[self.on, self.label[self.on]] = 1.0
        dz = g * (self.p - hot)
        off = g.abs() * (self.p * (self.rel + self.off_lse[:, None] + 4 * U32) + 2 * U32 * (self.p - hot).abs())
        H = torch.where(self.on[:, None], self.H, 0.0)
        rounding = 2.0 ** -23 if f32 else HALF[self.t]    # pieces: what the dropped products hold
        M = H.shape[0]
        self.dH, self.dW, self.db = dz @ self.W.T, H.T @ dz, dz.sum(0)

        def products(a, b, terms):
            return (a @ b) * (U32 * (terms + 4) * 1.3 + rounding)
        self.off_dH = off @ self.W.T.abs() + products(dz.abs() + off, self.W.T.abs(), N) + LEAST
        self.off_dW = H.T.abs() @ off + products(H.T.abs(), dz.abs() + off, M) + LEAST
        self.off_db = off.sum(0) + U32 * 130 * (dz.abs() + off).sum(0) + LEAST      # 64 rows a wavefront, then 64 bits
        return self
