"""Cases of the language-model operators that hold a training step's products
and its end: the gated feed-forward block, cross entropy straight from the
hidden states, and the gradients' norm and clipping.

Every case is a dict of plain values whose ``kind`` names the operator and its
direction:

  ffn         y = act(x Wg^T) (x Wu^T)
  ffn_grad    its gradients, those of the weights one per worker
  ce          cross entropy of the logits s h E^T of a token table E, the
              logits not kept: the loss alone, or with the gradients in h and
              (one per worker) in E
  norm        the global norm of every worker's gradients
  clip        that, and the gradients scaled to at most a norm, written into
              the workers' contributions to a collective

Types are "bf16", "f32" and "f64".  ``own`` chooses between the plain form and
the library's operators.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "f64": torch.float64}
MAX_NORM = 1.0


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def listed():
    return [
        # One decoding step of a small serving batch: the weights are read
        # once for 8 tokens.
        {"name": "ffn-decode", "kind": "ffn", "P": 1, "n": 8, "D": 4096, "F": 12288,
         "act": "silu", "type": "bf16"},
        # A prompt's or a training step's forward pass over 16,384 tokens.
        {"name": "ffn-train", "kind": "ffn", "P": 1, "n": 16384, "D": 4096, "F": 12288,
         "act": "silu", "type": "bf16"},
        # The backward pass of an ordinary step.
        {"name": "ffn-grad-train", "kind": "ffn_grad", "P": 1, "n": 8192, "D": 4096, "F": 12288,
         "act": "silu", "type": "bf16", "grad": "bf16"},
        # Eight workers of a small fp32 model, odd sizes throughout.
        {"name": "ffn-grad-workers", "kind": "ffn_grad", "P": 8, "n": 517, "D": 1001, "F": 2731,
         "act": "gelu", "type": "f32", "grad": "f32"},
        # A small model's last layer, a few sentences: latency.
        {"name": "ce-small", "kind": "ce", "P": 1, "n": 61, "D": 96, "V": 1003, "type": "f32",
         "grad": "f32", "scale": 1.0, "skip": 0.1},
        # Evaluation: the loss of 2,048 positions, no gradient.
        {"name": "ce-eval", "kind": "ce", "P": 1, "n": 2048, "D": 2048, "V": 32003,
         "type": "bf16", "grad": "none", "scale": 1.0, "skip": 0.0},
        # A large training step: 8,192 positions over 128,000 tokens.
        {"name": "ce-train", "kind": "ce", "P": 1, "n": 8192, "D": 4096, "V": 128000,
         "type": "bf16", "grad": "bf16", "scale": 1.0, "skip": 0.05},
        # Sixteen workers of a small bf16 model whose table gradients are
        # summed in fp32; an odd width and a scaled product.
        {"name": "ce-workers", "kind": "ce", "P": 16, "n": 517, "D": 250, "V": 5003,
         "type": "bf16", "grad": "f32", "scale": 0.5, "skip": 0.1},
        # The gradients of a very small model: latency.
        {"name": "clip-small", "kind": "clip", "P": 1, "layers": 2, "D": 96, "F": 250, "V": 1003,
         "type": "f32", "out": "f32"},
        # Monitoring: the norm of the bf16 gradients of 0.6e9 parameters.
        {"name": "norm-large", "kind": "norm", "P": 1, "layers": 24, "D": 1280, "F": 5120,
         "V": 32003, "type": "bf16", "out": "f32"},
        # The fp32 gradients of the same model, clipped into the contribution.
        {"name": "clip-train", "kind": "clip", "P": 1, "layers": 24, "D": 1280, "F": 5120,
         "V": 32003, "type": "f32", "out": "f32"},
        # Sixteen workers of a small model, fp64 contributions for the stale
        # allreduce, each worker clipped by its own norm; odd sizes.
        {"name": "clip-workers", "kind": "clip", "P": 16, "layers": 6, "D": 250, "F": 1001,
         "V": 5003, "type": "f32", "out": "f64"},
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["ffn", "ffn_grad", "ce", "ce", "norm", "clip"])
    t = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("norm", "clip"):
        P = _logint(rng, 1, 32) if rng.random() < 0.5 else 1
        D = _logint(rng, 16, 1280)
        case = {"kind": kind, "P": P, "layers": _logint(rng, 1, 24), "D": D,
                "F": _logint(rng, 2 * D, 4 * D), "V": _logint(rng, 50, 32003),
                "type": rng.choice(["bf16", "f32", "f32", "f64"])}
        while _elements(case) * P > 1 << 28 and case["P"] > 1:
            case["P"] = P = P // 2
        out = "f64" if case["type"] == "f64" else rng.choice(["f32", "f64", case["type"]])
        return {**case, "out": out}
    P = _logint(rng, 1, 16) if rng.random() < 0.4 else 1
    D = _logint(rng, 16, 4096)
    grad = rng.choice(["f32", t])
    if kind in ("ffn", "ffn_grad"):
        F = _logint(rng, 16, 12288)
        n = _logint(rng, 1, 8192)
        n = max(1, min(n, (1 << (38 if t == "bf16" else 36)) // (P * D * F), (1 << 27) // (P * F)))
        case = {"kind": kind, "P": P, "n": n, "D": D, "F": F,
                "act": rng.choice(["silu", "gelu"]), "type": t}
        return {**case, "grad": grad} if kind == "ffn_grad" else case
    V = _logint(rng, 60, 128000)
    V = min(V, (1 << 29) // (P * D))
    n = _logint(rng, 1, 8192)
    n = max(1, min(n, (1 << (40 if t == "bf16" else 37)) // (P * D * V), (1 << 29) // (P * V)))
    return {"kind": kind, "P": P, "n": n, "D": D, "V": V, "type": t,
            "grad": "none" if rng.random() < 0.25 else grad,
            "scale": rng.choice([1.0, 1.0, 0.125]), "skip": rng.choice([0.0, 0.1, 0.4])}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _shapes(c):
    """The parameters of a small transformer."""
    D, F = c["D"], c["F"]
    layer = [(D, D), (D, D), (D, D), (D, D), (F, D), (F, D), (D, F), (D,), (D,)]
    return [(c["V"], D)] + layer * c["layers"] + [(D,)]


def _elements(c):
    return sum(math.prod(s) for s in _shapes(c))


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind = case["kind"]
    t = TYPES[case["type"]]

    def normal(shape, scale, dtype=t):
        x = torch.randn(shape, device=DEV, generator=gen,
                        dtype=torch.float64 if dtype == torch.float64 else torch.float32)
        return x.mul_(scale).to(dtype)

    s = {"case": case}
    P = case["P"]
    if kind in ("ffn", "ffn_grad"):
        N, D, F = P * case["n"], case["D"], case["F"]
        s["x"] = normal((N, D), 1.0)
        s["w_gate"] = normal((F, D), 1.5 / math.sqrt(D))
        s["w_up"] = normal((F, D), 1.0 / math.sqrt(D))
        if kind == "ffn_grad":
            s["dy"] = normal((N, F), 0.01)
    elif kind == "ce":
        N, D, V = P * case["n"], case["D"], case["V"]
        s["table"] = normal((V, D), 1.0 / (case["scale"] * math.sqrt(D)))
        # tokens as vocabularies sorted by frequency have them; two of three
        # hidden states lean towards their token, as a trained model's do
        u = torch.rand(N, device=DEV, generator=gen)
        labels = ((V + 1.0) ** u).long().sub_(1).clamp_(0, V - 1)
        lean = 10.0 * torch.rand((N, 1), device=DEV, generator=gen)
        lean *= torch.rand((N, 1), device=DEV, generator=gen) < 0.66
        h = torch.randn((N, D), device=DEV, generator=gen)
        s["h"] = (h + lean * s["table"][labels].float() * case["scale"]).to(t)
        labels[torch.rand(N, device=DEV, generator=gen) < 0.03] = -100
        s["labels"] = labels.to(torch.int32)
        weight = torch.rand(N, device=DEV, generator=gen).add_(0.5).div_(N)
        weight[torch.rand(N, device=DEV, generator=gen) < case["skip"]] = 0.0
        s["weight"] = weight
    else:
        m = _elements(case)
        # each worker's norm lies between a fifth of the limit and five times
        # it, so that some are left alone
        size = torch.exp2(torch.rand(P, device=DEV, generator=gen) * 4.6 - 2.3)
        if P == 1:
            size = size.clamp_(min=1.5)
        s["grads"] = [(torch.randn((P,) + shape, device=DEV, generator=gen) *
                       (MAX_NORM * size / math.sqrt(m)).view((P,) + (1,) * len(shape))).to(t)
                      for shape in _shapes(case)]
        if kind == "clip":
            # the contributions, and each parameter's place in them
            s["flat"] = torch.empty((P, m), device=DEV, dtype=TYPES[case["out"]])
            sizes = [math.prod(shape) for shape in _shapes(case)]
            s["out"] = [v.unflatten(1, shape) for v, shape in
                        zip(s["flat"].split(sizes, 1), _shapes(case))]
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return OWN[kind](state["case"], state)
    return PLAIN[kind](state["case"], state)


def _own_ffn(c, s):
    from paper_2203_17063_amd import lm
    return lm.gated_ffn(s["x"], s["w_gate"], s["w_up"], act=c["act"])


def _own_ffn_grad(c, s):
    from paper_2203_17063_amd import lm
    return lm.gated_ffn_grad(s["x"], s["w_gate"], s["w_up"], s["dy"], act=c["act"], P=c["P"],
                             dtype=TYPES[c["grad"]])


def _own_ce(c, s):
    from paper_2203_17063_amd import lm
    if c["grad"] == "none":
        return lm.cross_entropy(s["h"], s["table"], s["labels"], s["weight"], scale=c["scale"],
                                grad=None)[0]
    loss, dh, dtable = lm.cross_entropy(s["h"], s["table"], s["labels"], s["weight"],
                                        scale=c["scale"], P=c["P"], dtype=TYPES[c["grad"]])
    return {"loss": loss, "dh": dh, "dtable": dtable}


def _own_norm(c, s):
    from paper_2203_17063_amd import lm
    return lm.grad_norm(s["grads"], P=c["P"])


def _own_clip(c, s):
    from paper_2203_17063_amd import lm
    norms = lm.clip_grads(s["grads"], MAX_NORM, P=c["P"], out=s["out"])
    return {"norms": norms, "contributions": s["flat"]}


OWN = {"ffn": _own_ffn, "ffn_grad": _own_ffn_grad, "ce": _own_ce, "norm": _own_norm,
       "clip": _own_clip}


def _act(kind, g):
    """The activation and its derivative."""
    if kind == "silu":
        q = 1.0 / (1.0 + torch.exp(-g))
        return g * q, q * (1.0 + g * (1.0 - q))
    c = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * c, c + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _ffn(c, s):
    x = s["x"].float()
    return (_act(c["act"], x @ s["w_gate"].float().t())[0] *
            (x @ s["w_up"].float().t())).to(TYPES[c["type"]])


def _ffn_grad(c, s):
    t, P, n = TYPES[c["type"]], c["P"], c["n"]
    x, dy, wg, wu = (s[k].float() for k in ("x", "dy", "w_gate", "w_up"))
    g, u = x @ wg.t(), x @ wu.t()
    a, da = _act(c["act"], g)
    dg, du = dy * u * da, dy * a

    def of_weights(d):
        return (d.view(P, n, -1).transpose(1, 2) @ x.view(P, n, -1)).to(TYPES[c["grad"]])

    return {"dx": (dg @ wg + du @ wu).to(t), "dw_gate": of_weights(dg), "dw_up": of_weights(du)}


def _ce(c, s):
    t, P, n = TYPES[c["type"]], c["P"], c["n"]
    h, table, w, y = s["h"].float(), s["table"].float(), s["weight"], s["labels"].long()
    known = (y >= 0) & (y < c["V"])
    y = y.clamp(0, c["V"] - 1)[:, None]
    w = torch.where(known, w, torch.zeros((), device=DEV))[:, None]
    z = (h * c["scale"]) @ table.t()
    z = z.sub_(z.amax(1, keepdim=True))
    at = z.gather(1, y)
    z = z.exp_()
    total = z.sum(1, keepdim=True)
    loss = (w * (torch.log(total) - at))[:, 0]
    if c["grad"] == "none":
        return loss
    z = z.mul_(w / total)
    z.scatter_add_(1, y, -w)
    dtable = z.view(P, n, -1).transpose(1, 2) @ (h * c["scale"]).view(P, n, -1)
    return {"loss": loss, "dh": ((z @ table) * c["scale"]).to(t),
            "dtable": dtable.to(TYPES[c["grad"]])}


def _norms(c, s):
    return torch.stack([g.double().square().view(c["P"], -1).sum(1)
                        for g in s["grads"]]).sum(0).sqrt()


def _clip(c, s):
    norms = _norms(c, s)
    by = (MAX_NORM / norms).clamp(max=1.0)[:, None]
    flat = torch.cat([(g.view(c["P"], -1) * by.to(wide(c))).to(TYPES[c["out"]])
                      for g in s["grads"]], 1)
    return {"norms": norms, "contributions": flat}


def wide(c):
    return torch.float64 if "f64" in (c["type"], c["out"]) else torch.float32


PLAIN = {"ffn": _ffn, "ffn_grad": _ffn_grad, "ce": _ce, "norm": _norms, "clip": _clip}


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    size = {"bf16": 2, "f32": 4, "f64": 8, "none": 0}
    kind, P, e = case["kind"], case["P"], size[case["type"]]
    if kind in ("ffn", "ffn_grad"):
        N, D, F = P * case["n"], case["D"], case["F"]
        if kind == "ffn":
            return {"bytes": (N * D + 2 * F * D + N * F) * e, "flops": 4.0 * N * D * F}
        # both projections again, then two products each for dx and the weights
        return {"bytes": (2 * N * D + 2 * F * D + N * F) * e + 2 * P * F * D * size[case["grad"]],
                "flops": 12.0 * N * D * F}
    if kind == "ce":
        N, D, V = P * case["n"], case["D"], case["V"]
        live = N * (1.0 - case["skip"]) * 0.97
        one = 2.0 * live * V * D
        if case["grad"] == "none":
            return {"bytes": live * D * e + V * D * e + 12 * N, "flops": one}
        return {"bytes": live * D * e + N * D * e + V * D * e +
                P * V * D * size[case["grad"]] + 12 * N, "flops": 3.0 * one}
    m = P * _elements(case)
    if kind == "norm":
        return {"bytes": m * e, "flops": 2.0 * m}
    return {"bytes": m * (e + size[case["out"]]), "flops": 3.0 * m}


# --------------------------------------------------------------------------
# the definitions, in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind, P = case["kind"], case["P"]
    if kind in ("norm", "clip"):
        norms = torch.linalg.vector_norm(
            torch.stack([torch.linalg.vector_norm(g.double().flatten(1), dim=1)
                         for g in s["grads"]]), dim=0)
        if kind == "norm":
            return norms
        by = torch.where(norms > MAX_NORM, MAX_NORM / norms, 1.0)
        flat = torch.cat([torch.einsum("pm,p->pm", g.double().flatten(1), by)
                          for g in s["grads"]], 1)
        return {"norms": norms, "contributions": flat}
    if kind in ("ffn", "ffn_grad"):
        act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[case["act"]]
        x, wg, wu = (s[k].double() for k in ("x", "w_gate", "w_up"))
        if kind == "ffn":
            return act(torch.mm(x, wg.t())) * torch.mm(x, wu.t())
        g = torch.mm(x, wg.t()).requires_grad_(True)
        u = torch.mm(x, wu.t()).requires_grad_(True)
        dg, du = torch.autograd.grad(act(g) * u, (g, u), s["dy"].double())
        own_rows = [slice(p * case["n"], (p + 1) * case["n"]) for p in range(P)]
        return {"dx": torch.addmm(torch.mm(dg, wg), du, wu),
                "dw_gate": torch.stack([torch.mm(dg[r].t(), x[r]) for r in own_rows]),
                "dw_up": torch.stack([torch.mm(du[r].t(), x[r]) for r in own_rows])}
    h, table = s["h"].double(), s["table"].double()
    y = s["labels"].long()
    known = (y >= 0) & (y < case["V"])
    w = s["weight"].double() * known
    losses, dh = [], []
    dtable = torch.zeros((P,) + table.shape, dtype=torch.float64, device=DEV)
    # rows of one worker at a time, in pieces
    step = max(1, (1 << 28) // case["V"])
    for p in range(P):
        for r in range(p * case["n"], (p + 1) * case["n"], step):
            rows = slice(r, min(r + step, (p + 1) * case["n"]))
            z = torch.mm(h[rows], table.t()) * case["scale"]
            lse = torch.logsumexp(z, 1)
            at = y[rows].clamp(0, case["V"] - 1)
            i = torch.arange(at.numel(), device=DEV)
            losses.append(w[rows] * (lse - z[i, at]))
            if case["grad"] != "none":
                q = torch.exp(z - lse[:, None])
                q[i, at] -= 1.0
                q *= (w[rows] * case["scale"])[:, None]
                dh.append(torch.mm(q, table))
                dtable[p] += torch.mm(q.t(), h[rows])
    if case["grad"] == "none":
        return torch.cat(losses)
    return {"loss": torch.cat(losses), "dh": torch.cat(dh), "dtable": dtable}
