"""Plain 64-bit forms of the gated feed-forward update and the bounds the kernels are held to."""
import math

import torch

U32 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
ACTS = ["silu", "gelu", "relu", "sigmoid"]


def act(name, g):
    """act(g), its derivative, and bounds of |second derivative| and |derivative| (both over all g)."""
    if name == "relu":
        return g.clamp_min(0.0), (g > 0).to(g.dtype)
    if name == "gelu":
        cdf = 0.5 * torch.special.erfc(-g / math.sqrt(2.0))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if name == "sigmoid" else (g * s, s * (1 + g * (1 - s)))


def forward(x, wg, wu, bg, bu, name):
    x, wg, wu = x.double(), wg.double(), wu.double()
    g, u = x @ wg, x @ wu
    if bg is not None:
        g = g + bg.double()
    if bu is not None:
        u = u + bu.double()
    return act(name, g)[0] * u, g, u


def backward(x, wg, wu, g, u, dp, name):
    x, wg, wu, g, u, dp = (v.double() for v in (x, wg, wu, g, u, dp))
    a, da = act(name, g)
    dg, du = dp * u * da, dp * a
    return dg @ wg.T + du @ wu.T, x.T @ dg, x.T @ du, dg.sum(0), du.sum(0), dg, du


def off_act(name, g):
    """Largest errors of act(g) and act'(g) as the kernels form them in float32 from an exact g (their formulas; rcp and
    exp2 within 2^-23 relative, the exponent rounded: 2^-23 (1 + |g|) of the exponential)."""
    g = g.double().abs()
    if name == "relu":
        return 0.0 * g, 0.0 * g
    if name == "gelu":
        # 1.5e-7 / 2 of the series, eight roundings of a sum of terms below 1, the exponential of g^2 / 2
        e = torch.exp(-0.5 * g * g)
        cdf = 0.75e-7 + 24 * U32 + 4 * U32 * (1 + g * g) * e
        return g * cdf + 2 * U32 * g, cdf + 0.4 * g * e * U32 * (8 + 4 * g * g) + 4 * U32
    s = 2 * U32 * (5 + g * torch.exp(-g))            # relative error of s, the exponent's share fading with s -> 1
    full = 2 * U32 * (5 + g)                         # on the side where s -> 0 it is exp(g) itself
    rel = torch.maximum(s, full)
    lo = torch.exp(-g)                               # min(s, 1 - s) <= exp(-|g|)
    if name == "sigmoid":
        return rel * torch.ones_like(g) * torch.clamp(lo + 6 * U32 / rel, max=1.0), 4 * rel * lo + 4 * U32
    return g * (rel * lo + 8 * U32) + 2 * U32 * g, rel * lo * (2 + g) + (8 * U32) * (1 + 2 * g)
