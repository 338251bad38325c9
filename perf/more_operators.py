"""The operators of an attention layer over sampled neighbours and of a classifier's loss - what each is measured on.

  attn         o[u] = sum over the edges e of row u of softmax(scale q[u] . k[v_e] + bias[bucket_e]) v[v_e], heads apart,
               key and value heads shared by groups of query heads; a bucket of -1 leaves its edge out
  attn_train   the same, then the gradients of Q, K, V and of the bias table
  loss         loss[i] = log sum_n exp z[i,n] - z[i, label_i] of the class scores z = H W + b, which are not kept;
               a label of -1 leaves its row out
  loss_train   the same, then the gradients of H, W and b

Rows of attention are nodes of a mini-batch's block, so sizes run from one node asked for online to the 512 K rows of a
products-shaped input layer; classes run from the 47 of that workload to a vocabulary of node IDs.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


# ------------------------------------------------------------------ cases
def listed():
    return [
        # One node asked for online, its sampled neighbours: launch and latency are all there is to it.
        dict(name="attn_one_node_bf16", kind="attn", rows=1, sources=16, fan=15, skew=False, heads=4, shared=1, width=64, dtype="bf16",
             buckets=0, one_array=True),
        # The seeds' own layer in evaluation at float32, relations of edges as buckets.
        dict(name="attn_seeds_f32", kind="attn", rows=8000, sources=91_331, fan=15, skew=False, heads=8, shared=1, width=32, dtype="f32",
             buckets=32, one_array=True),
        # The input layer of the headline block in evaluation: the most rows and neighbours, two query heads to a key head.
        dict(name="attn_input_layer_bf16", kind="attn", rows=512_345, sources=1_149_890, fan=5, skew=False, heads=4, shared=2, width=64,
             dtype="bf16", buckets=16, one_array=True),
        # A training step of the headline block's middle layer: forward and backward.
        dict(name="attn_train_middle_bf16", kind="attn_train", rows=91_331, sources=512_345, fan=10, skew=False, heads=8, shared=1,
             width=32, dtype="bf16", buckets=32, one_array=True),
        # All neighbours instead of sampled ones: rows of up to 18 000 edges beside rows of eight.
        dict(name="attn_train_all_neighbours_bf16", kind="attn_train", rows=65_536, sources=500_000, fan=8, skew=True, heads=4, shared=1,
             width=16, dtype="bf16", buckets=64, one_array=False),
        # Class scores straight from attention: heads of 47 columns, all on one key head, at float32.
        dict(name="attn_train_w47_f32", kind="attn_train", rows=8000, sources=91_331, fan=15, skew=False, heads=4, shared=4, width=47,
             dtype="f32", buckets=0, one_array=False),
        # One node's loss online, and a mini-batch of seeds in a training step of the headline workload.
        dict(name="loss_one_node_bf16", kind="loss", rows=1, width=256, classes=47, dtype="bf16", bias=True),
        dict(name="loss_train_seeds_f32", kind="loss_train", rows=8000, width=256, classes=47, dtype="f32", bias=True),
        # More classes, still few beside the rows: one node of each row's neighbourhood is told from 1000.
        dict(name="loss_train_c1000_bf16", kind="loss_train", rows=16_384, width=512, classes=1000, dtype="bf16", bias=True),
        # Odd everything at float32: classes that are no multiple of anything.
        dict(name="loss_train_c10007_f32", kind="loss_train", rows=4001, width=300, classes=10_007, dtype="f32", bias=True),
        # Pretraining by telling a node's ID: a vocabulary of 65 536, in evaluation and in a training step.
        dict(name="loss_vocabulary_bf16", kind="loss", rows=32_768, width=256, classes=65_536, dtype="bf16", bias=False),
        dict(name="loss_train_vocabulary_bf16", kind="loss_train", rows=8192, width=512, classes=65_536, dtype="bf16", bias=False),
    ]


def _log(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    kind = rng.choice(["attn", "attn_train", "attn_train", "loss", "loss_train", "loss_train"])
    c = dict(kind=kind, dtype=rng.choice(["f32", "bf16"]))
    if kind.startswith("attn"):
        shared, groups = rng.choice([1, 1, 2, 3, 4, 8]), rng.randint(1, 6)
        width = _log(rng, 1, 160)
        skew = rng.random() < 0.3
        # three at least in training: the gradients of a score that nothing competes with are 0 but for roundings
        fan = _log(rng, 1 if kind == "attn" else 3, 12 if skew else 40)
        # the edges and columns of the listed training step's (skewed rows are 10/3 of fan long on average)
        most = 91_331 * 10 * 256 // (fan * (4 if skew else 1) * max(64, shared * groups * width))
        rows = _log(rng, 1, max(1, min(500_000, most)))
        c |= dict(rows=rows, sources=max(1, round(rows * rng.uniform(0.5, 10))), fan=fan, skew=skew, heads=shared * groups, shared=shared,
                  width=width, buckets=rng.choice([0, 2, 8, 32, 100, 500]), one_array=rng.random() < 0.5)
    else:
        width, classes = _log(rng, 8, 1500), _log(rng, 2, 70_000)
        most = 8192 * 512 * 65_536 // (6 if c["dtype"] == "f32" else 1)
        c |= dict(width=width, classes=classes, rows=_log(rng, 1, max(1, min(70_000, most // (width * classes), 500_000_000 // classes))),
                  bias=rng.random() < 0.5)
    return c


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(g, dtype, *shape):
    return torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32).to(dtype)


def _degrees(case):
    """Edges of the rows, by rank: a sampler's fan-out, which a quarter of the nodes have not the neighbours for; or all
    neighbours of a heavy-tailed graph, the largest row fan * rows^0.7."""
    i = torch.arange(case["rows"], dtype=torch.int64)
    if case["skew"]:
        return (case["fan"] * (case["rows"] / (i + 1).double()) ** 0.7).floor().long()
    return torch.where(i % 4 == 3, (i // 4) % (case["fan"] + 1), case["fan"])


def prepare(case, seed):
    c, g = dict(case), _generator(seed)
    t, M = DTYPES[c["dtype"]], c["rows"]
    s = {"case": c}
    if c["kind"].startswith("loss"):
        F, N = c["width"], c["classes"]
        s["H"] = _normal(g, t, M, F)
        s["W"] = (2.0 * _normal(g, torch.float32, F, N) / math.sqrt(F)).to(t)
        s["b"] = 0.5 * _normal(g, torch.float32, N) if c["bias"] else None
        s["labels"] = torch.randint(0, N, (M,), generator=g, device=DEVICE, dtype=torch.int64)
        if M > 1:                                       # a tenth of the nodes has no label
            s["labels"][torch.rand(M, generator=g, device=DEVICE) < 0.1] = -1
        if c["kind"] == "loss_train":                   # a mean over the rows, with weights
            s["dloss"] = (0.5 + torch.rand(M, generator=g, device=DEVICE)) / M
        return s
    n, k = c["heads"] * c["width"], c["heads"] // c["shared"] * c["width"]
    degrees = _degrees(c).to(DEVICE)[torch.randperm(M, generator=g, device=DEVICE)]
    s["indptr"] = torch.cat((torch.zeros(1, dtype=torch.int64, device=DEVICE), degrees.cumsum(0))).int()
    E, S = int(s["indptr"][-1]), c["sources"]
    # some sources are neighbours of many
    s["indices"] = (torch.rand(E, generator=g, device=DEVICE, dtype=torch.float64) ** 1.5 * S).long().clamp(max=S - 1).int()
    s["Q"] = _normal(g, t, M, n)
    if c["one_array"]:                                  # both come out of one projection
        s["KV"] = _normal(g, t, S, 2 * k)
        s["K"], s["V"] = s["KV"][:, :k], s["KV"][:, k:]
    else:
        s["K"], s["V"] = (_normal(g, t, S, k) for _ in range(2))
    if c["buckets"]:
        s["bucket"] = torch.randint(0, c["buckets"], (E,), generator=g, device=DEVICE, dtype=torch.int32)
        s["bucket"][torch.rand(E, generator=g, device=DEVICE) < 0.1] = -1
        s["bias"] = _normal(g, torch.float32, c["buckets"], c["heads"])
    else:
        s["bucket"] = s["bias"] = None
    if c["kind"] == "attn_train":
        s["dO"] = _normal(g, t, M, n)
    if own:                                             # a program has one plan for every block, whatever it calls on it
        from paper_2409_14939_amd import binding as B
        parts = B.PLAN_ALL | B.PLAN_PERM if c["kind"] == "attn_train" else B.PLAN_FWD
        s["plan"] = B.fastgl_block_plan_create(s["indptr"], s["indices"], S, parts)
    return s


# ------------------------------------------------------------------ plain forms
def _plain_loss(s):
    c = s["case"]
    t, labels = DTYPES[c["dtype"]], s["labels"]
    h, w = s["H"].float(), s["W"].float()
    z = h @ w
    if s["b"] is not None:
        z = z + s["b"]
    most = z.amax(1, keepdim=True)
    lse = most[:, 0] + torch.log(torch.exp(z - most).sum(1))
    on = labels >= 0
    at = labels.clamp(min=0)[:, None]
    loss = torch.where(on, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    if c["kind"] == "loss":
        return [loss, lse]
    g = torch.where(on, s["dloss"], torch.zeros_like(lse))
    dz = torch.exp(z - lse[:, None]) * g[:, None]
    dz.scatter_add_(1, at, -g[:, None])
    out = [loss, lse, (dz @ w.T).to(t), (h.T @ dz).to(t)]
    return out + ([dz.double().sum(0).float()] if s["b"] is not None else [])


def _plain_attn(s):
    c = s["case"]
    t, M, S, heads, D = DTYPES[c["dtype"]], c["rows"], c["sources"], c["heads"], c["width"]
    kv, scale = heads // c["shared"], 1.0 / math.sqrt(c["width"])
    degrees = (s["indptr"][1:] - s["indptr"][:-1]).long()
    u, v = torch.repeat_interleave(torch.arange(M, device=DEVICE), degrees), s["indices"].long()
    if s["bucket"] is not None:                         # edges that are left out do not take part
        on = s["bucket"] >= 0
        u, v, bucket = u[on], v[on], s["bucket"][on].long()

    def to_heads(x):                                    # every query head sees the key head of its group
        return x.float().reshape(x.shape[0], kv, 1, D).expand(x.shape[0], kv, c["shared"], D).reshape(x.shape[0], heads, D)

    q, k, x = s["Q"].float().reshape(M, heads, D), to_heads(s["K"][v]), to_heads(s["V"][v])
    score = (q[u] * k).sum(2) * scale
    if s["bias"] is not None:
        score = score + s["bias"][bucket]
    most = torch.full((M, heads), -math.inf, device=DEVICE).scatter_reduce_(0, u[:, None].expand(-1, heads), score, "amax")
    e = torch.exp(score - most[u])
    total = torch.zeros(M, heads, device=DEVICE).index_add_(0, u, e)
    lse = most + torch.log(total)
    p = e / total[u]
    o = torch.zeros(M, heads, D, device=DEVICE).index_add_(0, u, p[:, :, None] * x)
    out = [o.reshape(M, heads * D).to(t), lse]
    if c["kind"] == "attn":
        return out
    do = s["dO"].float().reshape(M, heads, D)
    dp = (do[u] * x).sum(2)
    delta = torch.zeros(M, heads, device=DEVICE).index_add_(0, u, p * dp)
    ds = p * (dp - delta[u])
    dq = torch.zeros(M, heads, D, device=DEVICE).index_add_(0, u, (scale * ds)[:, :, None] * k)
    dk = torch.zeros(S, heads, D, device=DEVICE).index_add_(0, v, (scale * ds)[:, :, None] * q[u])
    dv = torch.zeros(S, heads, D, device=DEVICE).index_add_(0, v, p[:, :, None] * do[u])
    dk, dv = (y.reshape(S, kv, c["shared"], D).sum(2).reshape(S, kv * D).to(t) for y in (dk, dv))
    out += [dq.reshape(M, heads * D).to(t)] + ([torch.cat((dk, dv), 1)] if c["one_array"] else [dk, dv])
    if s["bias"] is not None:
        spread = 1024 * bucket + torch.arange(len(u), device=DEVICE) % 1024     # many edges to one sum are slow: first to 1024
        sums = torch.zeros(1024 * c["buckets"], heads, device=DEVICE, dtype=torch.float64).index_add_(0, spread, ds.double())
        out.append(sums.reshape(c["buckets"], 1024, heads).sum(1).float())
    return out


# ------------------------------------------------------------------ the framework's calls
def _own(s):
    from paper_2409_14939_amd import binding as B

    c = s["case"]
    if c["kind"].startswith("loss"):
        loss, lse = B.fastgl_loss_fwd(s["H"], s["W"], s["b"], s["labels"])
        if c["kind"] == "loss":
            return [loss, lse]
        want = ("dH", "dW", "db") if c["bias"] else ("dH", "dW")
        grads = B.fastgl_loss_bwd(s["H"], s["W"], s["b"], s["labels"], lse, s["dloss"], want=want)
        return [loss, lse] + [x for x in grads if x is not None]
    block = (s["indptr"], s["indices"])
    how = dict(heads=c["heads"], kv_heads=c["heads"] // c["shared"], bucket=s["bucket"], bias=s["bias"], plan=s["plan"])
    o, lse = B.fastgl_attn_fwd(*block, s["Q"], s["K"], s["V"], **how)
    if c["kind"] == "attn":
        return [o, lse]
    into = {}
    if c["one_array"]:                                  # the gradient of the one projection that K and V came from
        dkv = torch.empty_like(s["KV"])
        k = s["K"].shape[1]
        into = dict(dK=dkv[:, :k], dV=dkv[:, k:])
    dq, dk, dv, dbias = B.fastgl_attn_bwd(*block, s["Q"], s["K"], s["V"], s["dO"], **how, **into)
    out = [o, lse, dq] + ([dkv] if c["one_array"] else [dk, dv])
    return out + ([dbias] if c["buckets"] else [])


def run(state):
    if own:
        return _own(state)
    return _plain_loss(state) if state["case"]["kind"].startswith("loss") else _plain_attn(state)


# ------------------------------------------------------------------ floors
def work(case):
    c = case
    b, M = BYTES[c["dtype"]], c["rows"]
    if c["kind"].startswith("loss"):
        F, N = c["width"], c["classes"]
        bias = 4 * N if c["bias"] else 0
        if c["kind"] == "loss":
            return {"bytes": b * (M * F + F * N) + bias + 16 * M, "flops": 2 * M * F * N}
        # scores, dH and dW: scores that are not kept are formed twice
        return {"bytes": 2 * b * (M * F + F * N) + 2 * bias + 20 * M, "flops": 8 * M * F * N}
    E = int(_degrees(c).sum())
    n, k = c["heads"] * c["width"], c["heads"] // c["shared"] * c["width"]
    S = min(c["sources"], E)                            # rows that are a neighbour of none are not needed
    table = 4 * c["buckets"] * c["heads"]
    index = 4 * (M + 1) + E * (8 if c["buckets"] else 4) + table
    forward = {"bytes": index + b * (2 * M * n + 2 * S * k) + 4 * M * c["heads"], "flops": 4 * E * n}
    if c["kind"] == "attn":
        return forward
    # and Q, dO, K, V once more, dQ, dK, dV: five products for each edge beside the two of the forward pass
    return {"bytes": forward["bytes"] + b * (2 * M * n + 2 * c["sources"] * k) + table, "flops": 14 * E * n}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    M = c["rows"]
    if c["kind"].startswith("loss"):
        h, w, y = s["H"].double(), s["W"].double(), s["labels"]
        z = h @ w if s["b"] is None else torch.addmm(s["b"].double(), h, w)
        lse = torch.logsumexp(z, 1)
        row = torch.arange(M, device=DEVICE)[y >= 0]
        loss = torch.zeros_like(lse)
        loss[row] = lse[row] - z[row, y[row]]
        if c["kind"] == "loss":
            return [loss, lse]
        z.sub_(lse[:, None]).exp_()
        z[row, y[row]] -= 1
        z.mul_(((y >= 0) * s["dloss"].double())[:, None])
        return [loss, lse, z @ w.T, h.T @ z] + ([z.sum(0)] if c["bias"] else [])
    heads, D, S = c["heads"], c["width"], c["sources"]
    ends, degrees = s["indptr"].long(), torch.diff(s["indptr"].long())
    u, v = torch.repeat_interleave(degrees), s["indices"].long()
    head = torch.arange(heads, device=DEVICE) // c["shared"]
    by_source = torch.argsort(v, stable=True)
    ends_of = torch.cat((ends[:1], torch.bincount(v, minlength=S).cumsum(0)))

    def over(x, ends):                                  # sums of runs of edges, as differences of running sums
        x = torch.cat((torch.zeros_like(x[:1]), x.cumsum(0)))
        return x[ends[1:]] - x[ends[:-1]]

    grad = c["kind"] == "attn_train"
    q, k, x = (s[n].double().reshape(s[n].shape[0], -1, D) for n in ("Q", "K", "V"))
    do = s["dO"].double().reshape(M, heads, D) if grad else None
    outs = {n: [] for n in ("o", "lse", "dq", "dk", "dv", "db")}
    for h in range(heads):                              # a head at a time: 64 bits an element are much
        kh, xh, qh = k[:, int(head[h])][v], x[:, int(head[h])][v], q[:, h][u]
        z = torch.linalg.vecdot(qh, kh) / math.sqrt(D)
        if s["bias"] is not None:
            z = torch.where(s["bucket"] < 0, -math.inf, z + s["bias"].double()[s["bucket"].long(), h])
        e = z.exp()                                     # scores are a few tens at most
        total = over((e > 0).double(), ends).round()     # rows that nothing is left of
        norm = torch.where(total > 0, over(e, ends), 1.0)
        outs["lse"].append(torch.where(total > 0, norm.log(), -math.inf))
        p = e / norm[u]
        outs["o"].append(over(p[:, None] * xh, ends))
        if not grad:
            continue
        doh = do[:, h][u]
        dp = torch.linalg.vecdot(doh, xh)
        ds = p * (dp - over(p * dp, ends)[u])
        if s["bias"] is not None:
            outs["db"].append(torch.bincount(s["bucket"].long() + 1, weights=ds, minlength=c["buckets"] + 1)[1:])
        ds = ds / math.sqrt(D)
        outs["dq"].append(over(ds[:, None] * kh, ends))
        outs["dk"].append(over((ds[:, None] * qh)[by_source], ends_of))
        outs["dv"].append(over((p[:, None] * doh)[by_source], ends_of))
    got = [torch.stack(outs["o"], 1).flatten(1), torch.stack(outs["lse"], 1)]
    if grad:
        dk, dv = (torch.stack(outs[n], 1).reshape(S, -1, c["shared"], D).sum(2).flatten(1) for n in ("dk", "dv"))
        got += [torch.stack(outs["dq"], 1).flatten(1)] + ([torch.cat((dk, dv), 1)] if c["one_array"] else [dk, dv])
        got += [torch.stack(outs["db"], 1)] if c["buckets"] else []
    return got
