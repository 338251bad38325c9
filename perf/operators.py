"""The operators of a residual feed-forward block that stands next to the aggregation of a sampled GNN:
norm, dropout, gated feed-forward, and feature rows held in 8 bits - what each is measured on.

  norm    h = R + drop(X), y = h / sqrt(mean(h^2) + eps) * w per row: the forward pass to float32 / bfloat16
          rows, or to e4m3 rows with one float32 scale each; the gradients of X, R and w
  drop    y = [R +] X * keep / (1 - p), keep from a counter-based generator, no mask stored
  gated   P = act(X Wg + bg) * (X Wu + bu); the gradients of X, both weights and both biases
  gather  rows of an e4m3 table, by ID, back to float32 / bfloat16

Rows are nodes of a mini-batch's block and widths those of its layers, so sizes run from one node asked
for online to the 1.15 M rows of a products-shaped input layer.

The generator is Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy
as 1, 2, 3", SC 2011): key = the seed's two halves, counter = (column / 8, row, the offset's two halves);
the eight 16-bit halves of an answer, low half first, belong to eight consecutive columns, and an element stays
where its half is >= t = round(65536 p).  It is then multiplied by 65536 / (65536 - t).
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
EPS = 1e-6
E4M3_MOST = 448.0        # the largest finite e4m3 value
SCALE_LEAST = 2.0 ** -126


# ------------------------------------------------------------------ cases
def listed():
    return [
        # One node's hidden row in online inference: launch and latency are all there is to it.
        dict(name="norm_one_node_bf16", kind="norm", rows=1, width=256, dtype="bf16", residual=True, p=0.0),
        # Between two layers of a training step: the middle layer of the headline block, 512 K rows.
        dict(name="norm_residual_dropout_bf16", kind="norm", rows=512_000, width=256, dtype="bf16", residual=True, p=0.5),
        # Its gradient at the widest raw feature rows (602 floats: no multiple of 16 bytes).
        dict(name="norm_grad_f32_w602", kind="norm_grad", rows=115_000, width=602, dtype="f32", residual=True, p=0.1),
        # A finished layer's rows on their way into an 8-bit feature table, at the width of the papers graph.
        dict(name="norm_to_8_bits_bf16", kind="norm8", rows=400_003, width=128, dtype="bf16", residual=False, p=0.0),
        # Dropout of the input features of the headline block: 1.15 M rows of 100.
        dict(name="drop_input_f32_w100", kind="drop", rows=1_150_000, width=100, dtype="f32", residual=False, p=0.5),
        # Class scores of one mini-batch of seeds: short odd rows, launch-bound.
        dict(name="drop_residual_bf16_w47", kind="drop", rows=8000, width=47, dtype="bf16", residual=True, p=0.1),
        # One node through the block online: both weight matrices are read for one row.
        dict(name="gated_one_node_bf16", kind="gated", rows=1, width=256, hidden=1024, dtype="bf16", act="silu", bias=True,
             train=False),
        # Forward pass of a training step on the second layer's rows: little to contract, much to write.
        dict(name="gated_train_bf16_k256", kind="gated", rows=115_000, width=256, hidden=1024, dtype="bf16", act="silu",
             bias=True, train=True),
        # The backward pass of a wide block: four large products.
        dict(name="gated_grad_bf16_k1024", kind="gated_grad", rows=16_384, width=1024, hidden=4096, dtype="bf16", act="gelu",
             bias=True),
        # The backward pass at float32 on one mini-batch of seeds, hidden width 8/3 of 256: odd rows.
        dict(name="gated_grad_f32_h683", kind="gated_grad", rows=8000, width=256, hidden=683, dtype="f32", act="silu",
             bias=True),
        # The input features of a mini-batch out of a device table held in 8 bits.
        dict(name="gather_table_8_bits_bf16", kind="gather", rows=390_000, table=20_000_000, width=128, dtype="bf16"),
        # The neighbours of a few seeds.
        dict(name="gather_few_8_bits_f32", kind="gather", rows=1500, table=2_400_000, width=100, dtype="f32"),
    ]


def _log(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "norm8", "drop", "gated", "gated", "gated_grad", "gated_grad", "gather"])
    c = dict(kind=kind, dtype=rng.choice(["f32", "bf16"]))
    if kind == "gather":
        width = _log(rng, 1, 2048)
        c |= dict(rows=_log(rng, 1, min(500_000, 60_000_000 // width)), table=_log(rng, 1, min(20_000_000, 2_500_000_000 // width)),
                  width=width)
    elif kind.startswith("gated"):
        width, hidden = _log(rng, 8, 1500), _log(rng, 8, 5000)
        # what the largest listed case multiplies, float32 at a sixth of it
        most = 16_384 * 1024 * 4096 // (6 if c["dtype"] == "f32" else 1)
        c |= dict(width=width, hidden=hidden, rows=_log(rng, 1, min(130_000, max(1, most // (width * hidden)))),
                  act=rng.choice(["silu", "gelu", "relu", "sigmoid"]), bias=rng.random() < 0.5)
        if kind == "gated":
            c["train"] = rng.random() < 0.5
    else:
        width = _log(rng, 1, 8192)
        c |= dict(width=width, rows=_log(rng, 1, min(1_200_000, 110_000_000 // width)), residual=rng.random() < 0.5,
                  p=rng.choice([0.0, 0.1, 0.5, 0.9]) if kind != "drop" else rng.choice([0.1, 0.3, 0.5, 0.9]))
    return c


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(g, dtype, *shape):
    return torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32).to(dtype)


def _rng_state(seed):
    # a program's seed and how far it has come: both of more than 32 bits
    return torch.tensor([0x1234_5678_9ABC + 77 * seed, (1 << 33) + 3 * seed], dtype=torch.int64, device=DEVICE)


def prepare(case, seed):
    c, g = dict(case), _generator(seed)
    t, M, F = DTYPES[c["dtype"]], c["rows"], c["width"]
    s = {"case": c}
    if c["kind"] in ("norm", "norm8", "drop"):
        s["X"] = _normal(g, t, M, F)
        s["R"] = 2.0 * _normal(g, t, M, F) if c["residual"] else None      # the residual stream is the larger one
        s["rng"] = _rng_state(seed) if c["p"] > 0 else None
        if c["kind"] != "drop":
            s["w"] = 1.0 + 0.2 * _normal(g, torch.float32, F)
    elif c["kind"] == "norm_grad":
        s["S"] = 2.0 * _normal(g, t, M, F)                                   # what the forward pass kept
        s["rstd"] = torch.rsqrt(s["S"].double().square().mean(1) + EPS).float()
        s["w"] = 1.0 + 0.2 * _normal(g, torch.float32, F)
        s["dY"] = _normal(g, t, M, F)
        s["dS"] = _normal(g, t, M, F) if c["residual"] else None           # what comes down the residual stream
        s["rng"] = _rng_state(seed) if c["p"] > 0 else None
    elif c["kind"] in ("gated", "gated_grad"):
        N = c["hidden"]
        s["X"] = _normal(g, t, M, F)
        s["Wg"], s["Wu"] = ((_normal(g, torch.float32, F, N) / math.sqrt(F)).to(t) for _ in range(2))
        s["bg"], s["bu"] = (0.1 * _normal(g, torch.float32, N) if c["bias"] else None for _ in range(2))
        if c["kind"] == "gated_grad":
            s["G"], s["U"] = ((s["X"].float() @ s[w].float() + (s[b] if c["bias"] else 0.0)).to(t) for w, b in (("Wg", "bg"), ("Wu", "bu")))
            s["dP"] = _normal(g, t, M, N)
    else:
        R = c["table"]
        bits = torch.randint(0, 127, (R, F), generator=g, device=DEVICE, dtype=torch.uint8)     # every finite value ...
        bits += torch.randint(0, 2, (R, F), generator=g, device=DEVICE, dtype=torch.uint8) << 7    # ... of either sign
        s["Q"] = bits.view(torch.float8_e4m3fn)
        s["scale"] = torch.exp(_normal(g, torch.float32, R) - 6.0)
        s["ids"] = torch.randint(0, R, (M,), generator=g, device=DEVICE, dtype=torch.int64)
    return s


# ------------------------------------------------------------------ plain forms
def _words(row, block, state):
    """The four 32-bit words of every (row, block of columns), as int64."""
    mask = 0xFFFFFFFF
    k0, k1 = state[0] & mask, (state[0] >> 32) & mask
    n2, n3 = state[1] & mask, (state[1] >> 32) & mask
    x0, x1 = torch.broadcast_tensors(block, row)
    x2, x3 = n2.expand_as(x0), n3.expand_as(x0)

    def ten_rounds(x0, x1, x2, x3, k0, k1):
        for _ in range(10):
            a, b = x0 * 0xD2511F53, x2 * 0xCD9E8D57              # 64-bit products, modulo 2^64
            x0, x1, x2, x3 = ((b >> 32) & mask) ^ x1 ^ k0, b & mask, ((a >> 32) & mask) ^ x3 ^ k1, a & mask
            k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
        return x0, x1, x2, x3

    return ten_rounds(x0, x1, x2, x3, k0, k1)


def _threshold(p):
    return round(65536 * p)


def _keep(M, F, p, state):
    blocks = -(-F // 8)
    w = torch.stack(_words(torch.arange(M, device=DEVICE)[:, None], torch.arange(blocks, device=DEVICE)[None, :], state), -1)
    halves = torch.stack((w & 0xFFFF, w >> 16), -1).reshape(M, blocks * 8)
    return halves[:, :F] >= _threshold(p)


def _drop(x, p, state):
    if p == 0.0:
        return x
    t = _threshold(p)
    keep = _keep(*x.shape, p, state)
    return torch.where(keep, x * (65536.0 / (65536 - t) if t < 65536 else 0.0), torch.zeros((), dtype=x.dtype, device=DEVICE))


def _gate(act, g):
    """act(g) and its derivative."""
    if act == "relu":
        on = (g > 0).to(g.dtype)
        return g * on, on
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-g * math.sqrt(0.5))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-g))
    if act == "sigmoid":
        return sig, sig * (1.0 - sig)
    return g * sig, sig * (1.0 + g * (1.0 - sig))


def _plain(s):
    c = s["case"]
    t, kind = DTYPES[c["dtype"]], c["kind"]
    if kind == "drop":
        y = _drop(s["X"].float(), c["p"], s["rng"])
        return [(y if s["R"] is None else y + s["R"].float()).to(t)]
    if kind in ("norm", "norm8"):
        h = _drop(s["X"].float(), c["p"], s["rng"])
        if s["R"] is not None:
            h = h + s["R"].float()
        rstd = 1.0 / torch.sqrt(h.square().mean(1) + EPS)
        y = h * rstd[:, None] * s["w"]
        out = [rstd] if s["R"] is None and s["rng"] is None else [rstd, h.to(t)]
        if kind == "norm":
            return out + [y.to(t)]
        scale = (y.abs().amax(1) / E4M3_MOST).clamp(min=SCALE_LEAST)
        return out + [scale, (y / scale[:, None]).to(torch.float8_e4m3fn)]
    if kind == "norm_grad":
        n = s["S"].float() * s["rstd"][:, None]
        dy = s["dY"].float()
        d = dy * s["w"]
        d = s["rstd"][:, None] * (d - n * (d * n).mean(1, keepdim=True))
        if s["dS"] is not None:
            d = d + s["dS"].float()
        dx = _drop(d, c["p"], s["rng"])
        return [dx.to(t), d.to(t), (dy.double() * n.double()).sum(0).float()]
    if kind == "gated":
        g, u = s["X"].float() @ s["Wg"].float(), s["X"].float() @ s["Wu"].float()
        if c["bias"]:
            g, u = g + s["bg"], u + s["bu"]
        p = _gate(c["act"], g)[0] * u
        return [p.to(t), g.to(t), u.to(t)] if c["train"] else [p.to(t)]
    if kind == "gated_grad":
        x, dp = s["X"].float(), s["dP"].float()
        a, da = _gate(c["act"], s["G"].float())
        dg, du = dp * s["U"].float() * da, dp * a
        out = [(dg @ s["Wg"].float().T + du @ s["Wu"].float().T).to(t), (x.T @ dg).to(t), (x.T @ du).to(t)]
        return out + ([dg.double().sum(0).float(), du.double().sum(0).float()] if c["bias"] else [])
    return [(s["Q"][s["ids"]].float() * s["scale"][s["ids"]][:, None]).to(t)]


# ------------------------------------------------------------------ the framework's calls
def _own(s):
    from paper_2409_14939_amd import binding as B

    c = s["case"]
    kind = c["kind"]
    if kind == "drop":
        return [B.fastgl_dropout(s["X"], s["rng"], c["p"], residual=s["R"])]
    if kind == "norm":
        y, h, rstd = B.fastgl_norm_fwd(s["X"], s["w"], EPS, residual=s["R"], rng=s["rng"], p=c["p"])
        return [rstd, y] if h is None else [rstd, h, y]
    if kind == "norm8":
        q, scale, h, rstd = B.fastgl_norm_fwd_e4m3(s["X"], s["w"], EPS, residual=s["R"], rng=s["rng"], p=c["p"])
        return [rstd, scale, q] if h is None else [rstd, h, scale, q]
    if kind == "norm_grad":
        return list(B.fastgl_norm_bwd(s["S"], s["w"], s["rstd"], s["dY"], dS=s["dS"], rng=s["rng"], p=c["p"]))
    if kind == "gated":
        p, g, u = B.fastgl_gated_fwd(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], c["act"], want_GU=c["train"])
        return [p, g, u] if c["train"] else [p]
    if kind == "gated_grad":
        want = ("dX", "dWg", "dWu", "dbg", "dbu") if c["bias"] else ("dX", "dWg", "dWu")
        return [x for x in B.fastgl_gated_bwd(s["X"], s["Wg"], s["Wu"], s["G"], s["U"], s["dP"], c["act"], want=want) if x is not None]
    return [B.fastgl_gather_rows_e4m3(s["Q"], s["scale"], s["ids"], c["dtype"])]


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ floors
def work(case):
    c = case
    b, M, F, kind = BYTES[c["dtype"]], c["rows"], c["width"], c["kind"]
    if kind == "gather":
        return {"bytes": M * (8 + 4 + F * (1 + b)), "flops": M * F}
    if kind.startswith("gated"):
        N = c["hidden"]
        if kind == "gated":
            return {"bytes": b * (M * F + 2 * F * N + M * N * (3 if c["train"] else 1)), "flops": 4 * M * F * N}
        return {"bytes": b * (2 * M * F + 4 * F * N + 3 * M * N), "flops": 8 * M * F * N}
    extra = 1 if c["residual"] else 0
    if kind == "drop":
        return {"bytes": b * M * F * (2 + extra), "flops": 2 * M * F}
    if kind == "norm_grad":
        return {"bytes": b * M * F * (3 + extra + (1 if c["p"] > 0 else 0)) + 4 * M + 8 * F, "flops": 10 * M * F}
    kept = 1 if c["residual"] or c["p"] > 0 else 0
    out = M * F + 4 * M if kind == "norm8" else b * M * F
    return {"bytes": b * M * F * (1 + extra + kept) + out + 4 * M + 4 * F, "flops": 5 * M * F}


# ------------------------------------------------------------------ the definitions in 64 bits
def _mulhilo(a, m):
    """High and low word of the product of a (int64 < 2^32) and a 32-bit constant, from halves of 16 bits."""
    a1, a0, m1, m0 = a // 65536, a % 65536, m // 65536, m % 65536
    middle = a1 * m0 + a0 * m1 + (a0 * m0) // 65536          # < 2^34
    return a1 * m1 + middle // 65536, (middle % 65536) * 65536 + (a0 * m0) % 65536


def _exact_drop(x, p, seed, offset):
    if p == 0.0:
        return x
    M, F = x.shape
    t = round(65536 * p)
    out = torch.empty_like(x)
    low = 1 << 32
    step = max(1, (1 << 24) // F)
    for first in range(0, M, step):                       # some rows at a time: eight int64 an element are much
        last = min(M, first + step)
        i = torch.arange(first, last, device=DEVICE).reshape(-1, 1)
        j = torch.arange(F, device=DEVICE).reshape(1, -1)
        counter = [(j // 8 + 0 * i), (i + 0 * j), torch.full((last - first, F), offset % low, device=DEVICE),
                   torch.full((last - first, F), offset // low, device=DEVICE)]
        key = [seed % low, seed // low]
        for _ in range(10):
            h0, l0 = _mulhilo(counter[0], 0xD2511F53)
            h1, l1 = _mulhilo(counter[2], 0xCD9E8D57)
            counter = [h1 ^ counter[1] ^ key[0], l1, h0 ^ counter[3] ^ key[1], l0]
            key = [(key[0] + 0x9E3779B9) % low, (key[1] + 0xBB67AE85) % low]
        word = torch.where(j % 8 < 4, torch.where(j % 8 < 2, counter[0], counter[1]), torch.where(j % 8 < 6, counter[2], counter[3]))
        half = torch.where(j % 2 == 0, word % 65536, word // 65536)
        out[first:last] = torch.where(half >= t, x[first:last] * 65536.0 / max(1, 65536 - t), 0.0)
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    kind, p = c["kind"], c.get("p", 0.0)
    state = s["rng"].tolist() if s.get("rng") is not None else [0, 0]
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v) and k not in ("rng", "ids", "Q")}
    if kind == "gather":
        bits = s["Q"].view(torch.uint8)[s["ids"]].long()
        sign, e, m = 1 - 2 * (bits // 128), (bits // 8) % 16, bits % 8
        size = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.exp2(e.double() - 10))
        return [sign * size * d["scale"][s["ids"]].unsqueeze(1)]
    if kind == "drop":
        return [_exact_drop(d["X"], p, *state) + d.get("R", 0.0)]
    if kind in ("norm", "norm8"):
        h = _exact_drop(d["X"], p, *state) + d.get("R", 0.0)
        rms = ((h * h).sum(1) / c["width"] + EPS).sqrt()
        y = h / rms.unsqueeze(1) * d["w"]
        out = [1 / rms] + ([h] if c["residual"] or p > 0 else [])
        if kind == "norm":
            return out + [y]
        scale = (y.abs().max(1).values / 448).clamp_min(2.0 ** -126)
        z = y / scale.unsqueeze(1)
        # to the nearest of the multiples of 2^-9, or of an eighth of the power of two below the value
        step = torch.exp2(torch.floor(torch.log2(z.abs().clamp_min(2.0 ** -6))) - 3)
        return out + [scale, torch.round(z / step) * step]
    if kind == "norm_grad":
        n = d["S"] * d["rstd"].unsqueeze(1)
        t = d["dY"] * d["w"]
        g = (t - n * (t * n).sum(1, keepdim=True) / c["width"]) * d["rstd"].unsqueeze(1) + d.get("dS", 0.0)
        return [_exact_drop(g, p, *state), g, (d["dY"] * n).sum(0)]
    erf = torch.special.erf
    if kind == "gated":
        g = torch.addmm(d["bg"], d["X"], d["Wg"]) if c["bias"] else d["X"] @ d["Wg"]
        u = torch.addmm(d["bu"], d["X"], d["Wu"]) if c["bias"] else d["X"] @ d["Wu"]
    else:
        g, u = d["G"], d["U"]
    if c["act"] == "relu":
        a, da = g.clamp_min(0), (g > 0).double()
    elif c["act"] == "gelu":
        a = g * (1 + erf(g / math.sqrt(2))) / 2
        da = (1 + erf(g / math.sqrt(2))) / 2 + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    else:
        e = torch.sigmoid(g)
        a, da = (e, e * (1 - e)) if c["act"] == "sigmoid" else (g * e, e + g * e * (1 - e))
    if kind == "gated":
        return [a * u, g, u] if c["train"] else [a * u]
    dg, du = d["dP"] * u * da, d["dP"] * a
    out = [dg @ d["Wg"].T + du @ d["Wu"].T, d["X"].T @ dg, d["X"].T @ du]
    return out + ([dg.sum(0), du.sum(0)] if c["bias"] else [])
