"""fp32 products of the library one term at a time, for tests that see a lost
digit: every sum over rows or columns has one to three terms of full mantissas,
so that results are bounded by a few u = 2^-24 of themselves, and not by the
length of the sum.

A product of one term.  Of the nine products of an element's three bf16 pieces
the three smallest are left out, 2^-23 + 2^-32 of the term; the other six are
added from the smallest on, the last addition within 2 u (units that round or
cut off), those before it on sums of at most 2^-7 of the term: 4.1 u in all,
ONE below.  A further term adds 2 u of the sum's magnitude.  A product of pieces
that goes missing leaves up to 2^-16 (256 u), or 2^-8, of the term.

Each case is a dict of inputs; check() compares outputs with the exact ones, and
emulate() gives the outputs that the given products of pieces lead to (the rest
in 64 bits)."""
import math

import torch

F32, F64 = torch.float32, torch.float64
U = 2.0 ** -24
ONE = 5 * U
SIX = ((1, 1), (0, 2), (2, 0), (0, 1), (1, 0), (0, 0))


def _pieces(v):
    v = v.to(F32)
    hi = v.bfloat16().float()
    mid = (v - hi).bfloat16().float()
    lo = (v - hi - mid).bfloat16().float()
    return [p.double() for p in (hi, mid, lo)]


def pieces_product(a, b, which=SIX):
    """a @ b, rounded to fp32, from the products `which` of their pieces."""
    pa, pb = _pieces(a), _pieces(b)
    return sum(pa[i] @ pb[j] for i, j in which).to(F32)


def _full(shape, lo, hi, g):
    """Values of [lo, hi) with all 24 bits."""
    return (lo + (hi - lo) * torch.rand(shape, generator=g, dtype=F64)).to(F32)


# --------------------------------------------------------------------------
# the feed-forward block
# --------------------------------------------------------------------------

def ffn_case(P, n, D, F, dtype=F32):
    """x has one element other than zero in a row, of [5, 8), and wg lies in
    [4, 8), so that silu(g) = g and its slope is 1 (1 + exp(-20) is 1 in fp32).
    dy has one element in a row: dx has two terms, the weights' gradients one."""
    g = torch.Generator().manual_seed(n + 3 * D + 7 * F)
    N = P * n
    i = torch.arange(N)
    x, dy = torch.zeros((N, D)), torch.zeros((N, F))
    # (no two rows of a worker with both places alike, for D and F without a
    # common factor and n up to D F)
    x[i, i % D] = _full((N,), 5, 8, g)
    dy[i, i % F] = _full((N,), 1, 2, g)
    assert math.gcd(D, F) == 1 and n <= D * F
    c = {"x": x, "dy": dy, "wg": _full((F, D), 4, 8, g), "wu": _full((F, D), 1, 2, g)}
    # (what bf16 rounds up to 8 is still 20 or more with the others)
    return dict({k: v.to(dtype) for k, v in c.items()}, P=P)


def _per_worker(d, x, P, product):
    n = x.shape[0] // P
    return torch.stack([product(d[p * n:(p + 1) * n].t(), x[p * n:(p + 1) * n]) for p in range(P)])


def ffn_emulate(c, which=None):
    """y, dx, dw_gate and dw_up; which: the products of pieces of one stage, by
    the names of its results, where they are not all six."""
    which = which or {}

    def product(stage):
        return lambda a, b: pieces_product(a, b, which.get(stage, SIX))
    g, u = product("y")(c["x"], c["wg"].t()), product("y")(c["x"], c["wu"].t())
    # (backward, the projections are whole, so that its own products show)
    g0, u0 = (pieces_product(c["x"], c[k].t()) for k in ("wg", "wu"))
    dg, du = c["dy"].float() * u0, c["dy"].float() * g0
    dx = product("dx")(torch.cat([dg, du], 1), torch.cat([c["wg"], c["wu"]], 0))
    return {"y": g * u, "dx": dx, "dw_gate": _per_worker(dg, c["x"], c["P"], product("dw_gate")),
            "dw_up": _per_worker(du, c["x"], c["P"], product("dw_up"))}


def ffn_check(c, got):
    """The names of results that are off by more than their bounds: y by two
    products, two roundings; dg and du by a product and two roundings, 7 u; dx by
    theirs, a product and one more term; the weights' gradients by theirs and a
    product.  All terms are positive."""
    x, dy, wg, wu = (c[k].double() for k in ("x", "dy", "wg", "wu"))
    g, u = x @ wg.t(), x @ wu.t()
    dg, du = dy * u, dy * g
    want = {"y": (g * u, 2 * ONE + 2 * U), "dx": (dg @ wg + du @ wu, 7 * U + ONE + 2 * U),
            "dw_gate": (_per_worker(dg, x, c["P"], torch.matmul), 7 * U + ONE),
            "dw_up": (_per_worker(du, x, c["P"], torch.matmul), 7 * U + ONE)}
    return _outside(got, {k: (v, e * v) for k, (v, e) in want.items()})


def _outside(got, want):
    out = []
    for k in got:
        value, error = want[k]
        assert got[k].shape == value.shape, k
        off = (got[k].double().cpu() - value).abs()
        if not (off <= error + 2.0 ** -110).all():
            out.append((k, float((off / (error + 2.0 ** -110)).max())))
    return out


# --------------------------------------------------------------------------
# cross entropy
# --------------------------------------------------------------------------

def ce_loss_case(N, D, V):
    """h has one element other than zero in a row, and the first token's logit of
    16 or more is the largest, the others -16 or less, one of them the label's:
    the loss is the difference of two logits (the sum of exponentials is 1)."""
    g = torch.Generator().manual_seed(N + 3 * D + 7 * V)
    h = torch.zeros((N, D))
    h[torch.arange(N), torch.arange(N) % D] = _full((N,), 4, 8, g)
    table = -_full((V, D), 4, 8, g)
    table[0] *= -1
    return {"h": h, "table": table, "y": torch.randint(1, V, (N,), generator=g).to(torch.int32)}


def ce_loss_emulate(c, which=SIX):
    z = pieces_product(c["h"], c["table"].t(), which)
    return {"loss": z[:, 0] - z.gather(1, c["y"].long()[:, None])[:, 0]}


def ce_loss_check(c, got):
    """Each logit within a product and the scale's, which is 1; then a difference,
    the logarithm of 1 (the others add 2^-40), the weight."""
    z = c["h"].double() @ c["table"].double().t()
    want = z[:, 0] - z.gather(1, c["y"].long()[:, None])[:, 0]
    return _outside(got, {"loss": (want, (ONE + 4 * U) * want)})


# Logits of three tokens, in quarters, and of the others.
_FEW = (0.0, -0.5, -1.25)
_FAR = -40.0


def _softmax(c):
    """softmax - [label] and the bound of its error.  The logits are exact:
    column 0 of h and of the table, in quarters, are all that adds to them.
    Exponentials within 4 u, their sum (three that count, zeros) within 8 u,
    its inverse within 2 u, the product: p is within 16 u, its difference from the
    label's 1 rounded once more."""
    z = torch.outer(c["h"][:, 0].double(), c["table"][:, 0].double())
    p = torch.softmax(z, 1)
    hot = torch.zeros_like(p)
    known = c["y"] >= 0
    hot[known, c["y"][known].long()] = 1.0
    p[~known] = 0.0
    # (rows of bf16 take exponentials off by (1.2 |x| + 1) u of x = z, the largest
    # logit being 0)
    far = 1.2 * z.abs() if c["h"].dtype != F32 else 0.0
    return p - hot, (16 + far) * U * p + U * (p + hot)


def _ce_case(N, D, V, g):
    h, table = torch.zeros((N, D)), torch.zeros((V, D))
    h[:, 0] = torch.randint(3, 7, (N,), generator=g) / 4.0
    table[:, 0] = _FAR
    table[:3, 0] = torch.tensor(_FEW)
    return h, table, torch.randint(0, 3, (N,), generator=g).to(torch.int32)


def ce_dh_case(N, D, V):
    """dh has three terms, of table rows in [1, 2)."""
    g = torch.Generator().manual_seed(N + 3 * D + 7 * V)
    h, table, y = _ce_case(N, D, V, g)
    table[:, 1:] = _full((V, D - 1), 1, 2, g)
    return {"P": 1, "h": h, "table": table, "y": y}


def ce_dh_emulate(c, which=SIX):
    return {"dh": pieces_product(_softmax(c)[0].to(F32), c["table"], which)}


def ce_dh_check(c, got):
    dz, e = _softmax(c)
    table = c["table"].double()
    want = dz @ table
    return _outside(got, {"dh": (want, e @ table.abs() + (ONE + 5 * U) * (dz.abs() @ table.abs()))})


def ce_de_case(P, n, D, V, dtype=F32):
    """One row of each worker counts: dE has one term, of a hidden state in [1, 2)
    where the table is zero."""
    g = torch.Generator().manual_seed(P * n + 3 * D + 7 * V)
    h, table, y = _ce_case(P * n, D, V, g)
    h[:, 1:] = _full((P * n, D - 1), 1, 2, g)
    live = torch.arange(P) * n + torch.arange(P) * 5 % n
    keep = torch.zeros(P * n, dtype=torch.bool)
    keep[live] = True
    y[~keep] = -1
    return {"P": P, "h": h.to(dtype), "table": table.to(dtype), "y": y, "live": live}


def ce_de_emulate(c, which=SIX):
    dz = _softmax(c)[0].to(F32)[c["live"]]
    h = c["h"][c["live"]]
    return {"dtable": torch.stack([pieces_product(dz[p][:, None], h[p][None], which)
                                   for p in range(c["P"])])}


def ce_de_check(c, got):
    dz, e = (t[c["live"]] for t in _softmax(c))
    h = c["h"].double()[c["live"]]
    want = dz[:, :, None] * h[:, None]
    return _outside(got, {"dtable": (want, e[:, :, None] * h[:, None].abs() + ONE * want.abs())})
