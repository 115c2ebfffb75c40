"""Cases of the language-model operators: token embeddings, the residual joint
of a block with its norms, and distillation from a teacher's top logits.

Every case is a dict of plain values whose ``kind`` names the operator and its
direction:

  lookup      rows of a token table, scaled
  embed_grad  the table's gradient, one per worker, from one or two
              micro-batches (the second added to the first)
  norm        the joint after a block and before the next one:
              u = rms(f) (o + w_post), x' = a x + b g u, h = rms(x') (o + w_pre)
  norm_grad   its gradients
  distill     loss and logit gradients of a batch

Types are "bf16", "f32" and "f64".  ``own`` chooses between the plain form and
the library's operators.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "f64": torch.float64}
EPS = 1e-6


def wide(*types):
    """The type sums are held in: 32 bits, 64 where an operand has them."""
    return torch.float64 if torch.float64 in types else torch.float32


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def listed():
    return [
        # One decoding step of a small serving batch: latency.
        {"name": "lookup-decode", "kind": "lookup", "n": 8, "V": 128000, "D": 4096,
         "table": "bf16", "act": "bf16", "ids": "i64", "pad": 0.0},
        # The input end of a large training step: fp32 master table, bf16
        # activations.
        {"name": "lookup-train", "kind": "lookup", "n": 131072, "V": 128000, "D": 4096,
         "table": "f32", "act": "bf16", "ids": "i64", "pad": 0.05},
        # An ordinary step: 8,192 tokens in each of two micro-batches, a table
        # of no round size.
        {"name": "embed-grad-micro", "kind": "embed_grad", "P": 1, "n": 8192, "V": 32003,
         "D": 2048, "act": "bf16", "grad": "f32", "ids": "i64", "pad": 0.05, "micro": 2},
        # The largest: 131,072 tokens into a table of 128,000 rows.
        {"name": "embed-grad-large", "kind": "embed_grad", "P": 1, "n": 131072, "V": 128000,
         "D": 4096, "act": "bf16", "grad": "f32", "ids": "i64", "pad": 0.0, "micro": 1},
        # Sixteen workers of a small model, each with its own fp64 gradient
        # for the stale allreduce; odd sizes.
        {"name": "embed-grad-workers", "kind": "embed_grad", "P": 16, "n": 1031, "V": 5003,
         "D": 250, "act": "f32", "grad": "f64", "ids": "i32", "pad": 0.1, "micro": 1},
        # One decoding step of one sequence: latency.
        {"name": "norm-decode", "kind": "norm", "P": 1, "n": 1, "D": 8192, "act": "bf16",
         "w": "bf16", "gate": "none", "gate_rows": 1, "post": True, "pre": True, "b": 1.0},
        # The joint of a large model over 32,768 tokens, one gate per token.
        {"name": "norm-train", "kind": "norm", "P": 1, "n": 32768, "D": 8192, "act": "bf16",
         "w": "f32", "gate": "rows", "gate_rows": 1, "post": True, "pre": True, "b": 1.0},
        # Its gradients, ordinary: 8 sequences of 1,024 tokens, one gate per
        # sequence.
        {"name": "norm-grad-seq", "kind": "norm_grad", "P": 1, "n": 8192, "D": 4096,
         "act": "bf16", "w": "f32", "gate": "rows", "gate_rows": 1024, "post": True,
         "pre": True, "b": 1.0},
        # Gradients of eight workers of a small fp32 model, a learned gate per
        # channel, an odd width.
        {"name": "norm-grad-workers", "kind": "norm_grad", "P": 8, "n": 517, "D": 1001,
         "act": "f32", "w": "f32", "gate": "param", "gate_rows": 0, "post": True, "pre": True,
         "b": 0.5},
        # A small student: a thousand-word vocabulary, a few sentences.
        {"name": "distill-small", "kind": "distill", "N": 61, "V": 1003, "K": 8, "act": "f32",
         "tau": 1.0, "kd": 1.0, "ce": 0.0, "skip": 0.1, "tail": 0},
        # Few positions over a long vocabulary, soft and hard targets mixed.
        {"name": "distill-few-rows", "kind": "distill", "N": 24, "V": 200001, "K": 64,
         "act": "f32", "tau": 2.0, "kd": 0.7, "ce": 0.3, "skip": 0.0, "tail": 0},
        # A large training step: 16,384 positions, padded vocabulary.
        {"name": "distill-train", "kind": "distill", "N": 16384, "V": 131072, "K": 64,
         "act": "bf16", "tau": 2.0, "kd": 0.9, "ce": 0.1, "skip": 0.05, "tail": 72},
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["lookup", "embed_grad", "embed_grad", "norm", "norm_grad", "norm_grad",
                       "distill", "distill"])
    act = rng.choice(["bf16", "bf16", "f32", "f64"])
    if kind in ("lookup", "embed_grad"):
        V, D = _logint(rng, 50, 150000), _logint(rng, 8, 8192)
        P = _logint(rng, 1, 32) if kind == "embed_grad" and rng.random() < 0.4 else 1
        V = max(2, min(V, (1 << 28) // (P * D)))
        n = max(1, min(_logint(rng, 1, 131072), (1 << 28) // (P * D)))
        case = {"kind": kind, "n": n, "V": V, "D": D, "act": act,
                "ids": rng.choice(["i32", "i64"]), "pad": rng.choice([0.0, 0.05, 0.3])}
        if kind == "lookup":
            return {**case, "table": rng.choice(["f32", act])}
        return {**case, "P": P, "grad": "f64" if act == "f64" else rng.choice(["f32", "f64", act]),
                "micro": rng.randint(1, 2)}
    if kind in ("norm", "norm_grad"):
        D = _logint(rng, 16, 8192)
        P = _logint(rng, 1, 16) if rng.random() < 0.4 else 1
        gate = rng.choice(["none", "rows", "param"])
        g = 1
        if gate == "rows" and rng.random() < 0.7:
            g = _logint(rng, 1, 2048)
        n = max(1, min(_logint(rng, 1, 32768), (1 << (26 if act == "f64" else 27)) // (P * D)))
        n = max(1, n // g) * g if n >= g else n
        g = min(g, n)
        post = rng.random() < 0.8
        return {"kind": kind, "P": P, "n": n, "D": D, "act": act,
                "w": "f64" if act == "f64" else rng.choice(["f32", act]), "gate": gate,
                "gate_rows": 0 if gate == "param" else g, "post": post,
                "pre": not post or rng.random() < 0.8, "b": rng.choice([1.0, 0.5])}
    V = _logint(rng, 60, 200000)
    N = max(1, min(_logint(rng, 1, 16384), (1 << 29) // V))
    ce = rng.choice([0.0, 0.3])
    return {"kind": kind, "N": N, "V": V, "K": min(_logint(rng, 1, 256), max(1, V // 4)),
            "act": act, "tau": rng.choice([1.0, 2.0, 4.0]), "kd": 1.0 - ce, "ce": ce,
            "skip": rng.choice([0.0, 0.1]), "tail": rng.choice([0, V // 50])}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _tokens(gen, count, V, pad, kind):
    """Token numbers as vocabularies sorted by frequency have them (the chance
    of a token falls with its number), a share `pad` of them padding."""
    u = torch.rand(count, device=DEV, generator=gen)
    ids = ((V + 1.0) ** u).long().sub_(1).clamp_(0, V - 1)
    ids[torch.rand(count, device=DEV, generator=gen) < pad] = -1
    return ids.to(torch.int64 if kind == "i64" else torch.int32)


def prepare(case, seed):
    gen = _generator(seed)
    kind = case["kind"]

    def normal(shape, dtype, scale=1.0, shift=0.0):
        x = torch.randn(shape, device=DEV, generator=gen,
                        dtype=torch.float64 if dtype == torch.float64 else torch.float32)
        return (x * scale + shift).to(dtype)

    s = {"case": case}
    if kind == "lookup":
        s["table"] = normal((case["V"], case["D"]), TYPES[case["table"]], 0.02)
        s["ids"] = _tokens(gen, case["n"], case["V"], case["pad"], case["ids"])
        s["scale"] = math.sqrt(case["D"])
    elif kind == "embed_grad":
        N = case["P"] * case["n"]
        s["ids"] = [_tokens(gen, N, case["V"], case["pad"], case["ids"])
                    for _ in range(case["micro"])]
        s["dy"] = [normal((N, case["D"]), TYPES[case["act"]], 0.01) for _ in range(case["micro"])]
        s["scale"] = math.sqrt(case["D"])
    elif kind in ("norm", "norm_grad"):
        N, D, act, w = case["P"] * case["n"], case["D"], TYPES[case["act"]], TYPES[case["w"]]
        s["x"] = normal((N, D), act, 2.0)
        s["f"] = normal((N, D), act, 0.7)
        s["w_post"] = normal((D,), w, 0.1, 1.0) if case["post"] else None
        s["w_pre"] = normal((D,), w, 0.1, 1.0) if case["pre"] else None
        s["gate"] = None
        if case["gate"] == "rows":
            s["gate"] = normal((-(-N // case["gate_rows"]), D), act, 0.3, 0.5)
        elif case["gate"] == "param":
            s["gate"] = normal((D,), w, 0.3, 0.5)
        if kind == "norm_grad":
            s["dh"] = normal((N, D), act, 0.01) if case["pre"] else None
            s["dxo"] = normal((N, D), act, 0.01)
    else:
        N, V, K, act = case["N"], case["V"], case["K"], TYPES[case["act"]]
        live = V - case["tail"]
        # distinct entries of every row, in no order, the last few of some
        # rows missing
        gaps = torch.randint(1, max(2, live // K), (N, K), device=DEV, generator=gen)
        first = torch.randint(0, live, (N, 1), device=DEV, generator=gen)
        idx = (first + gaps.cumsum(1)) % live
        top = torch.randn((N, K), device=DEV, generator=gen).mul_(2.0)
        top = top.sort(dim=1, descending=True).values
        z = torch.randn((N, V), device=DEV, generator=gen, dtype=torch.float32)
        # the student half agrees with the teacher
        z.scatter_add_(1, idx, 1.5 * top + 4.0)
        z[:, live:] = -math.inf
        s["z"] = z.to(act)
        del z
        held = torch.randint((K + 1) // 2, K + 1, (N, 1), device=DEV, generator=gen)
        s["idx"] = torch.where(torch.arange(K, device=DEV) < held, idx, -1).to(torch.int32)
        s["top"] = top.to(torch.float64 if act == torch.float64 else torch.float32)
        labels = idx[:, 0].clone()
        labels[torch.rand(N, device=DEV, generator=gen) < 0.05] = -100
        s["labels"] = labels.to(torch.int32) if case["ce"] else None
        weight = torch.rand(N, device=DEV, generator=gen).add_(0.5)
        weight[torch.rand(N, device=DEV, generator=gen) < case["skip"]] = 0.0
        s["weight"] = weight
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return OWN[kind](state["case"], state)
    return PLAIN[kind](state["case"], state)


def _own_lookup(c, s):
    from paper_2203_17063_amd import lm
    return lm.embed_lookup(s["table"], s["ids"], scale=s["scale"], dtype=TYPES[c["act"]])


def _own_embed_grad(c, s):
    from paper_2203_17063_amd import lm
    index = lm.embed_index(s["ids"][0], c["V"], P=c["P"])
    grad = lm.embed_grad(index, s["dy"][0], scale=s["scale"], dtype=TYPES[c["grad"]])
    if c["micro"] == 2:
        index = lm.embed_index(s["ids"][1], c["V"], P=c["P"])
        lm.embed_grad(index, s["dy"][1], scale=s["scale"], grad=grad, accumulate=True)
    return grad


def _own_norm(c, s):
    from paper_2203_17063_amd import lm
    x, h = lm.norm_forward(s["x"], s["f"], w_post=s["w_post"], w_pre=s["w_pre"], gate=s["gate"],
                           gate_rows=c["gate_rows"], res_scale=0.9, branch_scale=c["b"], eps=EPS)
    return {"x": x, "h": h}


def _own_norm_grad(c, s):
    from paper_2203_17063_amd import lm
    return lm.norm_grad(s["x"], s["f"], s["dh"], s["dxo"], w_post=s["w_post"], w_pre=s["w_pre"],
                        gate=s["gate"], gate_rows=c["gate_rows"], res_scale=0.9,
                        branch_scale=c["b"], eps=EPS, P=c["P"], dtype=TYPES[c["w"]])


def _own_distill(c, s):
    from paper_2203_17063_amd import lm
    loss, grad = lm.distill(s["z"], s["top"], s["idx"], tau=c["tau"], kd_weight=c["kd"],
                            ce_weight=c["ce"], labels=s["labels"], weight=s["weight"])
    return {"loss": loss, "grad": grad}


OWN = {"lookup": _own_lookup, "embed_grad": _own_embed_grad, "norm": _own_norm,
       "norm_grad": _own_norm_grad, "distill": _own_distill}


def _lookup(c, s):
    t = wide(s["table"].dtype)
    held = (s["ids"] >= 0) & (s["ids"] < c["V"])
    rows = s["table"][s["ids"].long().clamp(0, c["V"] - 1)].to(t) * s["scale"]
    return torch.where(held[:, None], rows, torch.zeros((), dtype=t, device=DEV)).to(
        TYPES[c["act"]])


def _add_tokens(c, sums, ids, dy, scale):
    """Adds the tokens' rows to the rows (worker, token) of `sums`."""
    held = (ids >= 0) & (ids < c["V"])
    worker = torch.arange(ids.numel(), device=DEV) // c["n"]
    rows = worker * c["V"] + ids.long().clamp(0, c["V"] - 1)
    part = torch.where(held[:, None], dy.to(sums.dtype), torch.zeros((), dtype=sums.dtype,
                                                                    device=DEV))
    sums.index_add_(0, rows, part * scale)


def _embed_grad(c, s):
    t = wide(TYPES[c["grad"]])
    # a gradient of fewer than 32 bits is rounded after each micro-batch
    sums = torch.zeros((c["P"] * c["V"], c["D"]), dtype=t, device=DEV)
    _add_tokens(c, sums, s["ids"][0], s["dy"][0], s["scale"])
    grad = sums.to(TYPES[c["grad"]])
    if c["micro"] == 2:
        sums = grad.to(t)
        _add_tokens(c, sums, s["ids"][1], s["dy"][1], s["scale"])
        grad = sums.to(TYPES[c["grad"]])
    return grad.view(c["P"], c["V"], c["D"])


def _gate_rows(c, s, t):
    """The gate of every row, or None."""
    if s["gate"] is None:
        return None
    if c["gate"] == "param":
        return s["gate"].to(t)
    rows = torch.arange(s["x"].shape[0], device=DEV) // c["gate_rows"]
    return s["gate"].to(t)[rows]


def _norm(c, s):
    act = TYPES[c["act"]]
    t = wide(act)
    f = s["f"].to(t)
    u = f
    if c["post"]:
        u = f * torch.rsqrt((f * f).mean(1, keepdim=True) + EPS) * s["w_post"].to(t)
    g = _gate_rows(c, s, t)
    u = u * c["b"] if g is None else u * g * c["b"]
    x = s["x"].to(t) * 0.9 + u
    h = None
    if c["pre"]:
        h = (x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * s["w_pre"].to(t)).to(act)
    return {"x": x.to(act), "h": h}


def _norm_grad(c, s):
    act, t = TYPES[c["act"]], wide(TYPES[c["act"]])
    P, n, D, b = c["P"], c["n"], c["D"], c["b"]
    out = {"dw_pre": None, "dw_post": None, "dgate": None}
    d = s["dxo"].to(t)
    if c["pre"]:
        x, dh = s["x"].to(t), s["dh"].to(t)
        q = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
        x = x * q
        out["dw_pre"] = (dh * x).view(P, n, D).sum(1).to(TYPES[c["w"]])
        dh = dh * s["w_pre"].to(t)
        d = d + q * (dh - x * (dh * x).mean(1, keepdim=True))
    out["dx"] = (d * 0.9).to(act)
    f = s["f"].to(t)
    if c["post"]:
        k = torch.rsqrt((f * f).mean(1, keepdim=True) + EPS)
        f = f * k
    u = f * s["w_post"].to(t) if c["post"] else f
    g = _gate_rows(c, s, t)
    du = d * b if g is None else d * g * b
    if c["gate"] == "param":
        out["dgate"] = (d * u * b).view(P, n, D).sum(1).to(TYPES[c["w"]])
    elif c["gate"] == "rows":
        rows = torch.arange(P * n, device=DEV) // c["gate_rows"]
        out["dgate"] = torch.zeros(s["gate"].shape, dtype=t, device=DEV).index_add_(
            0, rows, d * u * b).to(act)
    if c["post"]:
        out["dw_post"] = (du * f).view(P, n, D).sum(1).to(TYPES[c["w"]])
        du = du * s["w_post"].to(t)
        du = k * (du - f * (du * f).mean(1, keepdim=True))
    out["df"] = du.to(act)
    return out


def _distill(c, s):
    act, t, tau, V = TYPES[c["act"]], wide(TYPES[c["act"]]), c["tau"], c["V"]
    zero = torch.zeros((), dtype=t, device=DEV)
    w = s["weight"].to(t)
    z = s["z"].to(t)
    z = z - z.amax(1, keepdim=True)
    # the teacher's distribution over its entries
    idx = s["idx"].long()
    held = (idx >= 0) & (idx < V)
    idx = idx.clamp(0, V - 1)
    top = torch.where(held, s["top"].to(t), zero - math.inf)
    most = top.amax(1, keepdim=True)
    p = torch.exp((top - torch.where(most == -math.inf, zero, most)) / tau)
    mass = p.sum(1, keepdim=True)
    some = mass > 0
    p = torch.where(some, p / torch.where(some, mass, zero + 1), zero)
    # soft targets
    e = torch.exp(z / tau)
    total = e.sum(1, keepdim=True)
    logq = z.gather(1, idx) / tau - torch.log(total)
    terms = torch.where(p > 0, p * (torch.log(torch.where(p > 0, p, zero + 1)) - logq), zero)
    loss = c["kd"] * tau * tau * terms.sum(1)
    grad = e * ((c["kd"] * tau) * some.to(t) / total)
    grad.scatter_add_(1, idx, p * (-c["kd"] * tau))
    if s["labels"] is not None:
        y = s["labels"].long()
        known = (y >= 0) & (y < V)
        y = y.clamp(0, V - 1)[:, None]
        e = torch.exp(z)
        total = e.sum(1, keepdim=True)
        logq = z.gather(1, y) - torch.log(total)
        loss = loss + c["ce"] * torch.where(known, -logq[:, 0], zero)
        grad += e * (c["ce"] * known.to(t)[:, None] / total)
        grad.scatter_add_(1, y, -c["ce"] * known.to(t)[:, None])
    loss = torch.where(w != 0, loss * w, zero)
    grad = torch.where((w != 0)[:, None], grad.mul_(w[:, None]), zero)
    return {"loss": loss, "grad": grad.to(act)}


PLAIN = {"lookup": _lookup, "embed_grad": _embed_grad, "norm": _norm, "norm_grad": _norm_grad,
         "distill": _distill}


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    size = {"bf16": 2, "f32": 4, "f64": 8, "i32": 4, "i64": 8}
    if kind == "lookup":
        n, D, V = case["n"], case["D"], case["V"]
        # the distinct rows that tokens of this distribution touch: row v
        # holds log((v+2)/(v+1)) / log(V+1) of them
        held = n * (1.0 - case["pad"])
        rows = sum(-math.expm1(held * math.log1p(-min(1 - 1e-12, math.log((v + 2) / (v + 1)) /
                                                      math.log(V + 1)))) for v in range(V))
        return {"bytes": n * size[case["ids"]] + rows * D * size[case["table"]] +
                n * D * size[case["act"]], "flops": held * D}
    if kind == "embed_grad":
        N, D = case["P"] * case["n"], case["D"]
        held = N * (1.0 - case["pad"])
        return {"bytes": case["micro"] * (N * size[case["ids"]] + held * D * size[case["act"]]) +
                case["P"] * case["V"] * D * size[case["grad"]],
                "flops": case["micro"] * held * D}
    if kind in ("norm", "norm_grad"):
        N, D, a, w = case["P"] * case["n"], case["D"], size[case["act"]], size[case["w"]]
        gate = -(-N // case["gate_rows"]) * D * a if case["gate"] == "rows" else 0
        weights = (case["post"] + case["pre"] + (case["gate"] == "param")) * D * w
        if kind == "norm":
            return {"bytes": (3 + case["pre"]) * N * D * a + gate + weights,
                    "flops": 12.0 * N * D}
        return {"bytes": (4 + 2 * case["pre"]) * N * D * a + 2 * gate +
                (1 + case["P"]) * weights, "flops": 30.0 * N * D}
    N, V, K, a = case["N"], case["V"], case["K"], size[case["act"]]
    read = N * (1.0 - case["skip"])
    wide_size = 8 if case["act"] == "f64" else 4
    return {"bytes": read * (V * a + K * (wide_size + 4)) + N * V * a +
            N * (4 + wide_size + (4 if case["ce"] else 0)),
            "flops": read * V * (8.0 if case["ce"] else 5.0)}


# --------------------------------------------------------------------------
# the definitions, in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "lookup":
        held = torch.nonzero((s["ids"] >= 0) & (s["ids"] < case["V"]))[:, 0]
        y = torch.zeros((case["n"], case["D"]), dtype=torch.float64, device=DEV)
        y[held] = torch.index_select(s["table"], 0, s["ids"][held].long()).double() * s["scale"]
        return y
    if kind == "embed_grad":
        # runs of equal tokens in sorted order: differences of running sums
        total = torch.zeros((case["P"] * case["V"], case["D"]), dtype=torch.float64, device=DEV)
        for ids, dy in zip(s["ids"], s["dy"]):
            at = torch.nonzero((ids >= 0) & (ids < case["V"]))[:, 0]
            keys, order = torch.sort((at // case["n"]) * case["V"] + ids[at].long())
            rows, runs = torch.unique_consecutive(keys, return_counts=True)
            if rows.numel():
                ends = torch.cumsum(runs, 0) - 1
                running = torch.cumsum(dy[at[order]].double(), 0)[ends]
                running[1:] = running[1:] - running[:-1].clone()
                total[rows] += running
        return total.mul_(s["scale"]).view(case["P"], case["V"], case["D"])
    if kind in ("norm", "norm_grad"):
        return _exact_norm(case, s)
    step = max(1, (1 << 28) // case["V"])
    losses, grads = [], []
    for r in range(0, case["N"], step):
        loss, grad = _exact_distill(case, s, slice(r, r + step))
        losses.append(loss)
        grads.append(grad)
    return {"loss": torch.cat(losses), "grad": torch.cat(grads)}


def _exact_norm(case, s):
    def leaf(v):
        return None if v is None else v.double().requires_grad_(case["kind"] == "norm_grad")

    N, D = s["x"].shape

    def rms(v):
        return v / (v.pow(2).sum(1, keepdim=True) / D + EPS).sqrt()

    x, f, wq, wp, g = (leaf(s[k]) for k in ("x", "f", "w_post", "w_pre", "gate"))
    if case["kind"] == "norm_grad":
        # parameters by worker, so that each worker's gradient is its own
        wq, wp = (None if v is None else v.detach().expand(case["P"], D).clone()
                  .requires_grad_(True) for v in (wq, wp))
        if case["gate"] == "param":
            g = g.detach().expand(case["P"], D).clone().requires_grad_(True)

    def per_row(v):
        if v.dim() == 2 and v.shape[0] == case["P"]:
            return v.repeat_interleave(case["n"], 0)
        return v

    branch = f
    if wq is not None:
        branch = rms(f) * per_row(wq)
    if g is not None:
        branch = branch * (per_row(g) if case["gate"] == "param" else
                           g.repeat_interleave(case["gate_rows"], 0)[:N])
    if case["kind"] == "norm":
        y = 0.9 * x + case["b"] * branch
        return {"x": y, "h": None if wp is None else rms(y) * wp}
    # the gradient at a given x': d(x') from both of its uses, then the
    # branch's and the residual's shares of it
    d = s["dxo"].double()
    out = {"dw_pre": None, "dw_post": None, "dgate": None}
    if wp is not None:
        gx, out["dw_pre"] = torch.autograd.grad(rms(x) * per_row(wp), (x, wp),
                                                s["dh"].double())
        d = d + gx
    wanted = [v for v in (f, wq, g) if v is not None]
    got = list(torch.autograd.grad(case["b"] * branch, wanted, d))
    out["dx"], out["df"] = 0.9 * d, got.pop(0)
    if wq is not None:
        out["dw_post"] = got.pop(0)
    if g is not None:
        out["dgate"] = got.pop(0)
    return out


def _exact_distill(case, s, rows):
    V, tau = case["V"], case["tau"]
    z = s["z"][rows].double().requires_grad_(True)
    idx = s["idx"][rows].long()
    held = (idx >= 0) & (idx < V)
    some = held.any(1, keepdim=True)
    top = s["top"][rows].double().masked_fill(~held, -math.inf).masked_fill(~some, 0.0)
    p = torch.softmax(top / tau, 1) * some
    logq = torch.log_softmax(z / tau, 1).gather(1, idx.clamp(0, V - 1))
    kl = (torch.xlogy(p, p) - torch.where(held, p * logq, 0.0)).sum(1)
    loss = case["kd"] * tau ** 2 * kl
    if s["labels"] is not None:
        y = s["labels"][rows].long()
        known = (y >= 0) & (y < V)
        nll = torch.logsumexp(z, 1) - z.gather(1, y.clamp(0, V - 1)[:, None])[:, 0]
        loss = loss + case["ce"] * torch.where(known, nll, 0.0)
    loss = loss * s["weight"][rows].double()
    grad, = torch.autograd.grad(loss.sum(), z)
    return loss.detach(), grad
