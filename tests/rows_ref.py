"""Plain 64-bit forms of the norm, the dropout and the e4m3 rows, and the bounds the kernels are held to."""
import numpy as np
import torch

U32 = 2.0 ** -24                                   # half a step of float32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MASK = np.uint64(0xFFFFFFFF)


def philox(c0, c1, c2, c3, k0, k1):
    """Philox 4x32, ten rounds, on uint64 arrays of 32-bit values."""
    x = [np.asarray(v, dtype=np.uint64) for v in np.broadcast_arrays(c0, c1, c2, c3)]
    k0, k1 = np.uint64(k0), np.uint64(k1)
    for _ in range(10):
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(q >> np.uint64(32)) ^ x[1] ^ k0, q & MASK, (p >> np.uint64(32)) ^ x[3] ^ k1, p & MASK]
        k0, k1 = (k0 + np.uint64(0x9E3779B9)) & MASK, (k1 + np.uint64(0xBB67AE85)) & MASK
    return x


def threshold(p):
    return round(65536 * p)


def keep(M, F, p, state):
    """bool [M, F]"""
    seed, offset = (int(v) & (2 ** 64 - 1) for v in state)
    blocks = -(-F // 8)
    w = philox(np.arange(blocks, dtype=np.uint64)[None, :], np.arange(M, dtype=np.uint64)[:, None],
               np.uint64(offset & 0xFFFFFFFF), np.uint64(offset >> 32), seed & 0xFFFFFFFF, seed >> 32)
    halves = np.stack([h for v in w for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))], -1).reshape(M, blocks * 8)
    return torch.from_numpy(halves[:, :F] >= threshold(p))


def drop_scale(p):
    t = threshold(p)
    return 65536.0 / (65536 - t) if t < 65536 else 0.0


def drop(x, p, state):
    if p == 0.0:
        return x
    return torch.where(keep(*x.shape, p, state), x * drop_scale(p), torch.zeros((), dtype=x.dtype))


def norm(x, w, eps, r=None, p=0.0, state=None):
    """(y, h, rstd) in float64"""
    h = drop(x.double(), p, state)
    if r is not None:
        h = h + r.double()
    rstd = 1.0 / torch.sqrt(h.square().mean(1) + eps)
    return h * rstd[:, None] * w.double(), h, rstd


def norm_grad(s, w, rstd, dy, ds=None, p=0.0, state=None):
    """(dx, dr, dw) in float64"""
    s, w, rstd, dy = (v.double() for v in (s, w, rstd, dy))
    n, t = s * rstd[:, None], dy * w
    d = rstd[:, None] * (t - n * (t * n).mean(1, keepdim=True))
    if ds is not None:
        d = d + ds.double()
    return drop(d, p, state), d, (dy * n).sum(0)


def chain(F):
    """Roundings on the way of a term through a row's sum: those of one lane's columns, then the tree."""
    lanes = 64 if F <= 1024 else 256
    return 8 * -(-F // (8 * lanes)) + 10


def norm_bounds(x, w, y, h, rstd, dtype, r=None, p=0.0):
    """Largest errors of (y before it is rounded, h, rstd)."""
    xs = x.double().abs() * (drop_scale(p) if p > 0 else 1.0)
    off_h = U32 * ((xs if p > 0 else 0.0) + (h.abs() if r is not None else 0.0)) * torch.ones_like(h)      # product, sum
    F = h.shape[1]
    # relative error of the mean of squares, from its terms, its sum and its divisor; a root halves it
    of_sum = (2 * (off_h * h.abs()).sum(1) / h.square().sum(1).clamp_min(1e-300) + (chain(F) + 3) * U32) / 2 + 3 * U32
    off_rstd = of_sum * rstd
    off_y = (off_h * rstd[:, None] * w.double().abs() + y.abs() * (of_sum[:, None] + 3 * U32)) * 1.01
    return off_y, off_h * 1.01, off_rstd * 1.01


def guarded(shape, dtype, fill, shift=0):
    """(buffer, its inner part of that shape): 64 elements of `fill` on either side, `shift` more in front."""
    n = int(np.prod(shape))
    buf = torch.full((n + 128 + shift,), fill, dtype=torch.float32, device="cuda").to(dtype)
    return buf, buf[64 + shift:64 + shift + n].view(shape)


def bands_intact(buf, inner, fill):
    start = inner.storage_offset()
    n = inner.numel()
    v = buf.float()
    return bool((v[:start] == fill).all()) and bool((v[start + n:] == fill).all())


def shifted(t, by=1):
    """The same values on the device, `by` elements past an aligned address."""
    buf = torch.empty(t.numel() + 8, dtype=t.dtype, device="cuda")
    out = buf[by:by + t.numel()].view(t.shape)
    out.copy_(t)
    return out
