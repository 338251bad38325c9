"""Attention over a block's edges in 64 bits, and the largest errors of the kernels' float32 arithmetic from the same inputs."""
import torch

U32 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


class Attention:
    """Forward and backward pass of one block; every per-edge array is [edges that take part, heads].  With it the bounds: a dot
    product of D float32 terms is off by (D + 2) u of the sum of its terms' sizes, a probability by its score's error and that of
    its exponential's argument, a sum of n terms by n u of its terms' sizes (each term's own error apart)."""

    def __init__(self, indptr, indices, Q, K, V, heads, kv_heads, scale, bucket=None, bias=None):
        ip = torch.as_tensor(indptr).long()
        degrees = ip[1:] - ip[:-1]
        u, v = torch.repeat_interleave(torch.arange(len(degrees)), degrees), torch.as_tensor(indices).long()
        on = torch.ones(len(u), dtype=torch.bool) if bucket is None else bucket >= 0
        if bias is not None:
            on &= bucket < bias.shape[0]
        self.on, self.u, self.v = on, u[on], v[on]
        self.rows, self.sources, self.heads, self.shared, self.scale = len(degrees), K.shape[0], heads, heads // kv_heads, scale
        self.D = Q.shape[1] // heads
        self.bucket = None if bias is None else bucket[on].long()
        self.buckets = 0 if bias is None else bias.shape[0]
        u, v = self.u, self.v
        self.q = Q.double().reshape(self.rows, heads, self.D)
        self.k, self.x = (t.double().reshape(self.sources, kv_heads, self.D).repeat_interleave(self.shared, 1) for t in (K, V))
        ku, qu = self.k[v], self.q[u]
        dot, size = (ku * qu).sum(2) * scale, (ku * qu).abs().sum(2) * abs(scale)
        b = 0.0 if bias is None else bias.double()[self.bucket]
        s = dot + b
        self.most = torch.full((self.rows, heads), -torch.inf, dtype=torch.float64).scatter_reduce_(0, u[:, None].expand(-1, heads), s, "amax")
        safe = torch.where(self.most == -torch.inf, 0.0, self.most)
        e = torch.exp(s - safe[u])
        total = self.to_rows(e)
        self.lse = torch.where(total > 0, safe + torch.log(total), -torch.inf)
        self.p = torch.where(e > 0, e / total[u], 0.0)
        self.O = self.to_rows(self.p[:, :, None] * self.x[v])
        # scores: the dot product, the factor's rounding, the bias to powers of two and its addition
        self.n = torch.bincount(u, minlength=self.rows).double()[:, None]
        ok = torch.where(torch.isfinite(s), s, 0.0)
        off = U32 * ((self.D + 4) * size + 3 * (torch.as_tensor(b).abs().clamp(max=1e30) if bias is not None else 0.0) + 2 * ok.abs())
        # an exponential: its argument's rounding and two units of its own
        self.off_s = off + U32 * (4 + 2 * ok.abs() + 2 * torch.where(torch.isfinite(self.lse), self.lse, 0.0).abs()[u])
        worst = torch.zeros(self.rows, heads, dtype=torch.float64).scatter_reduce_(0, u[:, None].expand(-1, heads), self.off_s, "amax")
        self.off_row = worst
        self.off_lse = worst + U32 * (self.n + 8 + 4 * torch.where(torch.isfinite(self.lse), self.lse, 0.0).abs())
        self.off_O = (2 * worst + U32 * (self.n + 12))[:, :, None] * self.to_rows(self.p[:, :, None] * self.x[v].abs())

    def to_rows(self, x):
        return torch.zeros(self.rows, *x.shape[1:], dtype=torch.float64).index_add_(0, self.u, x)

    def to_sources(self, x):
        x = torch.zeros(self.sources, *x.shape[1:], dtype=torch.float64).index_add_(0, self.v, x)
        return x.reshape(self.sources, -1, self.shared, self.D).sum(2)

    def to_buckets(self, x):
        return torch.zeros(self.buckets, self.heads, dtype=torch.float64).index_add_(0, self.bucket, x)

    def backward(self, dO):
        """Sets dQ, dK, dV, dbias and off_ of each, for the kernels' own lse."""
        u, v = self.u, self.v
        g = dO.double().reshape(self.rows, self.heads, self.D)
        gu, xv, kv, qu = g[u], self.x[v], self.k[v], self.q[u]
        dp, size = (gu * xv).sum(2), (gu * xv).abs().sum(2)
        delta = self.to_rows(self.p * dp)
        ds = self.p * (dp - delta[u])
        self.ds = ds
        self.dQ = self.scale * self.to_rows(ds[:, :, None] * kv)
        self.dK, self.dV = self.scale * self.to_sources(ds[:, :, None] * qu), self.to_sources(self.p[:, :, None] * gu)
        off_p = self.off_s + self.off_lse[u]                       # relative
        off_dp = U32 * (self.D + 2) * size
        n = U32 * (self.n + 8)
        off_delta = self.to_rows(self.p * (dp.abs() * off_p + off_dp)) + n * self.to_rows(self.p * dp.abs())
        # dQ from the sums of p dp k and of p k
        k1 = kv.abs()
        first = self.to_rows((self.p * (dp.abs() * (off_p + n[u]) + off_dp))[:, :, None] * k1)
        pk = self.to_rows(self.p[:, :, None] * k1)
        second = self.to_rows((self.p * (off_p + n[u]))[:, :, None] * k1) * delta.abs()[:, :, None] + off_delta[:, :, None] * pk
        self.off_dQ = abs(self.scale) * (first + second + 4 * U32 * delta.abs()[:, :, None] * pk) + 4 * U32 * self.dQ.abs()
        off_ds = self.p * (off_p * (dp - delta[u]).abs() + off_dp + off_delta[u] + 2 * U32 * (dp.abs() + delta.abs()[u])) + 2 * U32 * ds.abs()
        m = torch.bincount(v, minlength=self.sources).double()[v][:, None] * self.shared + 8
        self.off_dK = abs(self.scale) * self.to_sources((off_ds + U32 * m * ds.abs())[:, :, None] * qu.abs()) + 4 * U32 * self.dK.abs()
        self.off_dV = self.to_sources((self.p * (off_p + U32 * m))[:, :, None] * gu.abs())
        if self.buckets:
            self.dbias = self.to_buckets(ds)
            # a workgroup's tables: float32 sums of its edges' share, then of its tables
            self.off_dbias = self.to_buckets(off_ds) + U32 * (len(u) / 100 + 300) * self.to_buckets(ds.abs())
        return self
