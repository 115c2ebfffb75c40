"""Distillation from a teacher's top logits through the library's call, loss
and gradient, against the definition in 64 bits.

Tolerances.  u = 2^-24 for fp32 sums (2^-53 for fp64).  An exponential of
argument -x is within (x + 4) u relative (the argument is rounded, the power
of two is within 2 u); a probability is an exponential over a sum of
exponentials, each as exact as its size lets it be: with every |argument| up
to X, softmax values are within (2 X + 64) u relative (64 for the additions
in a chain: up to 32 logits per thread and group, rescalings, lanes, waves,
parts).  A loss is a sum of K terms p (log p - log q), each within (2 X + 64)
u of p (|log p| + |log q| + 1).  Stored bf16 gradients add 2^-8 relative."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from gpu_common import announce                           # noqa: E402

pytestmark = pytest.mark.gpu

F64, F32, BF16 = torch.float64, torch.float32, torch.bfloat16
ULP = {F64: 2.0 ** -53, F32: 2.0 ** -24, BF16: 2.0 ** -8}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def _lm():
    from paper_2203_17063_amd import lm
    return lm


def _inputs(N, V, K, act, seed=0, top_type=F32, labels=True, weight=True, absent=0.2):
    g = torch.Generator().manual_seed(1000 * seed + N + V + K)
    z = torch.randn((N, V), generator=g, dtype=F64) * 2.5
    idx = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(N)]) if N else \
        torch.zeros((0, K), dtype=torch.int64)
    top = torch.randn((N, K), generator=g, dtype=F64) * 2.0
    z.scatter_add_(1, idx, top + 3.0)
    idx[torch.rand((N, K), generator=g) < absent] = -1
    y = torch.randint(-1, V, (N,), generator=g)
    w = torch.rand((N,), generator=g) + 0.5
    w[torch.rand((N,), generator=g) < 0.2] = 0.0
    return dict(z=z.to(act), top=top.to(top_type), idx=idx.to(torch.int32),
                labels=y.to(torch.int32) if labels else None, weight=w if weight else None)


def _reference(s, tau, kd, ce):
    """Loss, gradient and bounds of their errors in units of u, row by row."""
    z = s["z"].double()
    N, V = z.shape
    loss, grad = torch.zeros(N, dtype=F64), torch.zeros((N, V), dtype=F64)
    el, eg = torch.zeros(N, dtype=F64), torch.zeros((N, V), dtype=F64)
    for r in range(N):
        w = float(s["weight"][r]) if s["weight"] is not None else 1.0
        if w == 0.0:
            continue
        finite = z[r][torch.isfinite(z[r])]
        X = float((finite.max() - finite.min()) * max(1.0, 1.0 / tau)) if finite.numel() else 0.0
        k = 2 * X + 64
        held = [j for j in range(s["idx"].shape[1]) if 0 <= int(s["idx"][r, j]) < V
                and float(s["top"][r, j]) != -math.inf] if kd else []
        if held:
            i = s["idx"][r, held].long()
            t = s["top"][r, held].double()
            k = k + 2 * float((t.max() - t.min()) / tau)
            p = torch.softmax(t / tau, 0)
            logq = torch.log_softmax(z[r] / tau, 0)
            live = p > 0
            terms = torch.where(live, p * (torch.log(p) - logq[i]), torch.zeros((), dtype=F64))
            loss[r] += kd * tau * tau * terms.sum()
            mass = torch.where(live, p * (torch.log(p).abs() + logq[i].abs() + 1),
                               torch.zeros((), dtype=F64))
            el[r] += abs(kd) * tau * tau * k * mass.sum()
            gr = torch.exp(logq)
            eg[r] += abs(kd) * tau * k * gr
            eg[r].index_add_(0, i, abs(kd) * tau * k * p)
            gr.index_add_(0, i, -p)
            grad[r] += kd * tau * gr
        y = int(s["labels"][r]) if s["labels"] is not None and ce else -1
        if 0 <= y < V:
            logq = torch.log_softmax(z[r], 0)
            loss[r] -= ce * logq[y]
            el[r] += abs(ce) * k * (logq[y].abs() + 1)
            gr = torch.exp(logq)
            eg[r] += abs(ce) * k * gr
            eg[r, y] += abs(ce) * k
            gr[y] -= 1
            grad[r] += ce * gr
        loss[r] *= w
        grad[r] *= w
        el[r] *= abs(w)
        eg[r] *= abs(w)
    return loss, grad, el, eg


def _within(got, want, bound_u, acc, out_type):
    got = got.cpu().double()
    u = 2.0 ** -53 if acc == F64 else 2.0 ** -24
    # (the smallest fp32 numbers are flushed to zero)
    tol = bound_u * u + ULP[out_type] * (want.abs() + bound_u * u) + (
        0 if acc == F64 else 2.0 ** -120)
    bad = ~((got - want).abs() <= tol) & ~(got == want)
    assert not bad.any(), (int(bad.sum()),
                           float(((got - want).abs() / tol.clamp_min(1e-300)).max()))


def _check(s, tau=1.0, kd=1.0, ce=0.0, **kw):
    act = s["z"].dtype
    d = {k: v.cuda() if torch.is_tensor(v) else v for k, v in s.items()}
    loss, grad = _lm().distill(tau=tau, kd_weight=kd, ce_weight=ce, **d, **kw)
    want_l, want_g, el, eg = _reference(s, tau, kd, ce)
    acc = F64 if act == F64 else F32
    assert loss.dtype == acc and grad.dtype == act
    _within(loss, want_l, el, acc, acc)
    _within(grad, want_g, eg, acc, act)
    again = _lm().distill(tau=tau, kd_weight=kd, ce_weight=ce, **d)
    assert torch.equal(loss, again[0]) and torch.equal(grad, again[1])
    alone, none = _lm().distill(tau=tau, kd_weight=kd, ce_weight=ce, grad=None, **d)
    assert none is None and torch.equal(alone, loss)
    return loss, grad


MIXES = [(1.0, 1.0, 0.0), (2.0, 0.7, 0.3), (1.0, 0.5, 0.5), (3.5, 0.0, 1.0), (0.7, -0.5, 1.5)]


@pytest.mark.parametrize("act", [BF16, F32, F64])
@pytest.mark.parametrize("tau,kd,ce", MIXES)
@pytest.mark.parametrize("N,V,K", [(1, 1, 1), (1, 2, 1), (3, 7, 3), (9, 64, 5), (5, 1003, 70),
                                   (4, 4099, 64), (2, 8200, 256)])
def test_small(act, tau, kd, ce, N, V, K):
    announce("distill", act, tau, kd, ce, N, V, K)
    _check(_inputs(N, V, K, act), tau, kd, ce)


@pytest.mark.parametrize("act,N,V", [(BF16, 600, 20011), (F32, 600, 9001), (F64, 530, 5003),
                                     (BF16, 513, 33333)])
def test_many_rows(act, N, V):
    """More rows than the device runs at once, a workgroup each."""
    announce("distill, many rows", act, N, V)
    _check(_inputs(N, V, 16, act), 2.0, 0.7, 0.3)
    _check(_inputs(N, V, 16, act, labels=False), 1.5)


@pytest.mark.parametrize("act", [BF16, F32, F64])
@pytest.mark.parametrize("N,V", [(1, 200001), (3, 50021), (40, 16384), (7, 24577), (1, 700001)])
def test_few_rows(act, N, V):
    """Rows split over workgroups, entries in every part."""
    announce("distill, few rows", act, N, V)
    _check(_inputs(N, V, 33, act), 2.0, 0.7, 0.3)
    _check(_inputs(N, V, 33, act, labels=False), 1.0)


@pytest.mark.parametrize("act,V", [(BF16, 131072), (BF16, 150003), (F32, 90001), (F64, 40001)])
def test_long_rows_whole(act, V):
    """Rows longer than a workgroup's registers hold."""
    lm = _lm()
    announce("distill, long rows", act, V)
    s = _inputs(2, V, 20, act, weight=False)
    # as many rows as keep them whole; two different ones
    wide = {k: (v.repeat(*([300] + [1] * (v.dim() - 1))) if torch.is_tensor(v) else v)
            for k, v in s.items()}
    d = {k: v.cuda() if torch.is_tensor(v) else v for k, v in wide.items()}
    loss, grad = lm.distill(tau=2.0, kd_weight=0.7, ce_weight=0.3, **d)
    want_l, want_g, el, eg = _reference(s, 2.0, 0.7, 0.3)
    acc = F64 if act == F64 else F32
    for r in (0, 1, 598, 599):
        _within(loss[r], want_l[r % 2], el[r % 2], acc, acc)
        _within(grad[r], want_g[r % 2], eg[r % 2], acc, act)
    assert torch.equal(loss.view(300, 2), loss[:2].expand(300, 2))
    assert all(torch.equal(grad[r], grad[r % 2]) for r in range(0, 600, 37))


@pytest.mark.parametrize("top_type", [F64, F32, BF16])
@pytest.mark.parametrize("K", [0, 1, 63, 65, 1000, 1024])
def test_entries(top_type, K):
    announce("distill, entries", top_type, K)
    _check(_inputs(4, 3001, K, F32, top_type=top_type), 2.0, 0.7, 0.3)
    _check(_inputs(2, 40001, K, BF16, top_type=top_type), 1.0, 1.0, 0.0)


def test_rows_without_anything():
    """No entry, only entries outside the vocabulary or of -infinity, no label,
    weight 0 over logits that are NaN: zeros, exactly."""
    lm = _lm()
    for act, V in ((F32, 500), (BF16, 40000)):
        announce("distill, empty rows", act, V)
        s = _inputs(6, V, 4, act, weight=False, absent=0.0)
        s["idx"][0] = torch.tensor([-1, V, -5, 2 ** 31 - 1], dtype=torch.int32)
        s["top"][1] = -math.inf
        s["top"][2, 1:] = -math.inf
        s["weight"] = torch.tensor([1, 1, 1, 0, 1, 1], dtype=F32)
        s["z"][3] = float("nan")
        s["labels"] = torch.tensor([-1, V, 3, 3, -100, 2], dtype=torch.int32)
        loss, grad = _check(s, 2.0, 0.7, 0.3)
        assert not loss[[0, 1, 3]].any() and not grad[[0, 1, 3]].any()
        assert loss[4] != 0 and loss[5] != 0
        loss, grad = lm.distill(s["z"].cuda(), s["top"].cuda(), s["idx"].cuda(), kd_weight=0.0,
                                weight=s["weight"].cuda())
        assert not loss.any() and not grad.any()


def test_entries_named_twice():
    announce("distill, entries named twice")
    for N, V in ((5, 300), (2, 30001)):
        s = _inputs(N, V, 12, F32, absent=0.0)
        s["idx"][:, 3] = s["idx"][:, 0]
        s["idx"][:, 7] = s["idx"][:, 0]
        s["idx"][:, 11] = s["idx"][:, 5]
        s["labels"][:] = s["idx"][:, 0]
        _check(s, 2.0, 0.7, 0.3)


def test_masked_logits():
    """Parts of the vocabulary masked with -infinity and with the type's lowest
    value; a row of nothing but the lowest value is uniform; an entry that the
    student has masked costs an infinite loss and a finite gradient."""
    lm = _lm()
    for act, V in ((F32, 700), (BF16, 30000), (F64, 900)):
        announce("distill, masked logits", act, V)
        s = _inputs(4, V, 6, act, absent=0.0, weight=False)
        s["idx"] = s["idx"] % (V // 2)
        s["labels"] = s["labels"] % (V // 2)
        s["z"][0, V // 2:] = -math.inf
        s["z"][1, V // 2:] = torch.finfo(act).min
        s["z"][2, : V // 2 - 1:2] = s["z"][2, : V // 2 - 1:2]
        d = {k: v.cuda() if torch.is_tensor(v) else v for k, v in s.items()}
        loss, grad = lm.distill(tau=2.0, kd_weight=0.7, ce_weight=0.3, **d)
        cut = dict(s, z=s["z"][:2, : V // 2].contiguous(), top=s["top"][:2], idx=s["idx"][:2],
                   labels=s["labels"][:2])
        want_l, want_g, el, eg = _reference(cut, 2.0, 0.7, 0.3)
        acc = F64 if act == F64 else F32
        _within(loss[:2], want_l, el, acc, acc)
        _within(grad[:2, : V // 2], want_g, eg, acc, act)
        assert not grad[:2, V // 2:].any()
        low = torch.full((1, V), torch.finfo(act).min, dtype=act)
        one = dict(z=low, top=s["top"][:1], idx=s["idx"][:1], labels=s["labels"][:1], weight=None)
        _check(dict(one, z=torch.zeros((1, V), dtype=act)), 2.0, 0.7, 0.3)
        got = lm.distill(low.cuda(), d["top"][:1], d["idx"][:1], 2.0, 0.7, 0.3, d["labels"][:1])
        zero = lm.distill(torch.zeros_like(low).cuda(), d["top"][:1], d["idx"][:1], 2.0, 0.7, 0.3,
                          d["labels"][:1])
        assert torch.equal(got[0], zero[0]) and torch.equal(got[1], zero[1])
        hidden = s["z"].clone()
        hidden[3, s["idx"][3, 2].long()] = -math.inf
        loss, grad = lm.distill(hidden.cuda(), d["top"], d["idx"], 2.0)
        assert torch.isinf(loss[3]) and torch.isfinite(loss[:3]).all()
        assert torch.isfinite(grad[3]).all()


def test_large_logits():
    """Logits of thousands, where exp alone would overflow."""
    announce("distill, large logits")
    for V in (300, 20000):
        s = _inputs(4, V, 6, F32)
        s["z"] = s["z"] * 300.0 + 5000.0
        _check(s, 2.0, 0.7, 0.3)


def test_nan_stays_in_its_row():
    lm = _lm()
    announce("distill, NaN")
    for V in (300, 20000):
        s = _inputs(3, V, 6, F32, weight=False, absent=0.0)
        s["z"][1, 17] = float("nan")
        loss, grad = lm.distill(s["z"].cuda(), s["top"].cuda(), s["idx"].cuda())
        assert torch.isnan(loss[1]) and torch.isnan(grad[1]).all()
        assert torch.isfinite(loss[[0, 2]]).all() and torch.isfinite(grad[[0, 2]]).all()


def test_strides_and_in_place():
    """Logits as a view of a wider buffer at any element; the gradient in
    their place, and beside."""
    lm = _lm()
    for act, N, V in ((BF16, 7, 1001), (F32, 3, 20001), (BF16, 600, 2049)):
        announce("distill, strides", act, N, V)
        s = _inputs(N, V, 9, act)
        d = {k: v.cuda() if torch.is_tensor(v) else v for k, v in s.items()}
        want = lm.distill(tau=2.0, kd_weight=0.7, ce_weight=0.3, **d)
        wide = torch.full((N, V + 6), 5.0, dtype=act, device="cuda")
        view = wide[:, 3:3 + V]
        view.copy_(d["z"])
        d["z"] = view
        out = torch.full((N, V + 1), 5.0, dtype=act, device="cuda")
        got = lm.distill(tau=2.0, kd_weight=0.7, ce_weight=0.3, grad=out[:, 1:], **d)
        assert torch.equal(got[0], want[0]) and torch.equal(out[:, 1:], want[1])
        got = lm.distill(tau=2.0, kd_weight=0.7, ce_weight=0.3, grad=view, **d)
        assert torch.equal(got[0], want[0]) and torch.equal(view, want[1])
        assert (wide[:, :3] == 5).all() and (wide[:, 3 + V:] == 5).all() and (out[:, 0] == 5).all()


def test_no_rows_and_batches():
    lm = _lm()
    announce("distill, no rows")
    z = torch.empty((0, 50), device="cuda")
    loss, grad = lm.distill(z, torch.empty((0, 3), device="cuda"),
                            torch.empty((0, 3), dtype=torch.int32, device="cuda"))
    assert loss.shape == (0,) and grad.shape == (0, 50)
    s = _inputs(6, 80, 4, F32)
    d = {k: v.cuda() for k, v in s.items()}
    want = lm.distill(ce_weight=1.0, **d)
    got = lm.distill(ce_weight=1.0, **{k: v.view(2, 3, *v.shape[1:]) for k, v in d.items()})
    assert got[0].shape == (2, 3) and torch.equal(got[0].view(6), want[0])
    assert torch.equal(got[1].view(6, 80), want[1])


@pytest.mark.parametrize("N,V", [(3, 12), (1, 20000)])
def test_gradient_against_differences(N, V):
    """Central differences of the summed loss in 64 bits along random
    directions."""
    lm = _lm()
    announce("distill, differences", N, V)
    s = _inputs(N, V, 5, F64)
    d = {k: v.cuda() if torch.is_tensor(v) else v for k, v in s.items()}
    kw = dict(tau=1.7, kd_weight=0.7, ce_weight=0.3)
    _, grad = lm.distill(**d, **kw)
    for j in range(4):
        g = torch.Generator().manual_seed(200 + j)
        v = torch.randn((N, V), generator=g, dtype=F64).cuda()
        t = 1e-4
        up = lm.distill(**dict(d, z=d["z"] + t * v), grad=None, **kw)[0].sum()
        down = lm.distill(**dict(d, z=d["z"] - t * v), grad=None, **kw)[0].sum()
        exact = float((grad * v).sum())
        assert abs(float(up - down) / (2 * t) - exact) <= 1e-6 * (abs(exact) + 1.0)


def test_on_another_stream_and_in_a_graph():
    lm = _lm()
    for N, V in ((520, 1003), (3, 30011)):
        announce("distill, stream and graph", N, V)
        s = _inputs(N, V, 8, BF16)
        d = {k: v.cuda() for k, v in s.items()}
        kw = dict(tau=2.0, kd_weight=0.7, ce_weight=0.3)
        want = lm.distill(**d, **kw)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = lm.distill(**d, **kw)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = lm.distill(**d, **kw)
        for k in range(3):
            d["z"].copy_(_inputs(N, V, 8, BF16, seed=k + 1)["z"])
            graph.replay()
            torch.cuda.synchronize()
            want = lm.distill(**d, **kw)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals():
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("distill refusals")
    z, dz = torch.zeros((4, 16), device="cuda"), torch.zeros((4, 16), device="cuda")
    top, idx = torch.zeros((4, 3), device="cuda"), torch.zeros((4, 3), dtype=torch.int32,
                                                             device="cuda")
    loss, work = torch.zeros(4, device="cuda"), torch.zeros(64, device="cuda")

    def desc(**kw):
        d = dict(N=4, V=16, K=3, type=E.ECC_F32, top_type=E.ECC_F32, pad=0, d_z=z.data_ptr(),
                 ld_z=16, d_top=top.data_ptr(), d_idx=idx.data_ptr(), d_labels=None,
                 d_weight=None, tau=1.0, kd_weight=1.0, ce_weight=0.0)
        d.update(kw)
        return E.ecc_distill_t(**d)

    def status(a, d_loss=loss, d_dz=dz, ld=16, d_work=work):
        with pytest.raises(E.EccError) as e:
            E.ecc_distill(a, d_loss, d_dz, ld, d_work)
        return e.value.status

    E.ecc_distill(desc(), loss, dz, 16, work)
    for bad in (dict(N=-1), dict(V=0), dict(K=-1), dict(K=1025), dict(type=3), dict(top_type=4),
                dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")), dict(tau=float("inf")),
                dict(ld_z=15), dict(d_z=None), dict(d_top=None), dict(d_idx=None),
                dict(d_z=z.data_ptr() + 2), dict(d_idx=idx.data_ptr() + 1)):
        assert status(desc(**bad)) == E.ECC_ERR_ARG, bad
        assert E.ecc_distill_work_size(desc(**bad)) == -1
    assert status(desc(V=1 << 31, ld_z=1 << 31)) == E.ECC_ERR_RANGE
    assert status(desc(N=1 << 31)) == E.ECC_ERR_RANGE
    assert status(desc(), d_loss=None) == E.ECC_ERR_ARG
    assert status(desc(), d_work=None) == E.ECC_ERR_ARG
    assert status(desc(), d_work=work.data_ptr() + 4) == E.ECC_ERR_ARG
    assert status(desc(), ld=15) == E.ECC_ERR_ARG
    assert status(desc(), d_dz=z[1:]) == E.ECC_ERR_ARG
    assert status(desc(), d_dz=top) == E.ECC_ERR_ARG
    assert status(desc(), d_loss=dz) == E.ECC_ERR_ARG
    assert status(desc(), d_work=dz) == E.ECC_ERR_ARG
    # what the tensors say
    for args in ((z, top[:3], idx), (z, top, idx[:, :2]), (z.t(), top, idx)):
        with pytest.raises(ValueError):
            lm.distill(*args)
    for args in ((z.half(), top, idx), (z, top.half(), idx), (z, top, idx.long())):
        with pytest.raises(TypeError):
            lm.distill(*args)
    for kw in (dict(labels=idx[:, 0].long()), dict(weight=loss.double()), dict(weight=loss[:3]),
               dict(grad=dz[:3]), dict(loss=loss[:3]), dict(labels=idx[:, 0])):
        with pytest.raises(ValueError):
            lm.distill(z, top, idx, **kw)


def _same(a, b):
    return torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("act", [BF16, F32, F64])
@pytest.mark.parametrize("N,V", [(3, 40), (4, 1003), (2, 30001), (520, 2100)])
@pytest.mark.parametrize("tau", [1.0, 2.0, 4.0, 3.5, 0.5])
def test_rows_of_one_large_value(act, N, V, tau):
    """A row of one value is uniform, however large the value: as a row of zeros
    gives.  Teachers' rows alike."""
    lm = _lm()
    announce("distill, rows of one large value", act, N, V, tau)
    s = _inputs(N, V, 6, act, weight=False, absent=0.0, top_type=F64 if act == F64 else F32)
    d = {k: v.cuda() if torch.is_tensor(v) else v for k, v in s.items()}
    kw = dict(tau=tau, kd_weight=0.7, ce_weight=0.3)
    z = torch.zeros_like(d["z"])
    flat = torch.zeros_like(d["top"])
    want, want_flat = lm.distill(**dict(d, z=z), **kw), lm.distill(**dict(d, top=flat), **kw)
    assert all(torch.isfinite(v).all() for v in want + want_flat)
    for value in ((-1e20, -1e30, -1e100, -1e305, 1e20, 1e200) if act == F64 else
                  (-1e8, -1e10, -1e15, -1e30, -1e36, 1e10, 1e20, 1e30)):
        got = lm.distill(**dict(d, z=torch.full_like(z, value)), **kw)
        assert _same(got, want), value
        got = lm.distill(**dict(d, top=torch.full_like(flat, value)), **kw)
        assert _same(got, want_flat), value


@pytest.mark.parametrize("act", [F32, F64])
@pytest.mark.parametrize("tau,ce", [(1.0, 0.3), (2.0, 0.3), (4.0, 0.3), (3.5, 0.3), (1.5, 0.0)])
@pytest.mark.parametrize("N,V", [(3, 300), (2, 3001), (2, 30001)])
def test_logits_at_a_large_offset(act, tau, ce, N, V):
    """Logits spread over some tens around offsets of any size (all of them
    multiples of what the type resolves there), so that maxima of threads and
    parts lie on both sides of any limit within a row."""
    announce("distill, large offsets", act, tau, ce, N, V)
    g = torch.Generator().manual_seed(7)
    for at in ((2 ** k / 1.4426950408889634 * t for k in (10, 17, 19, 20, 21) for t in (1.0, tau))
               if act == F32 else
               (float(2 ** k) * t for k in (20, 45, 47, 49) for t in (1.0, tau))):
        step = 2.0 ** max(-10, math.ceil(math.log2(at)) - (23 if act == F32 else 50))
        most = int(30 / step)
        for sign in (1.0, -1.0):
            s = _inputs(N, V, 6, act, weight=False, absent=0.0)
            z = torch.randint(-most, most + 1, (N, V), generator=g, dtype=F64) * step
            offset = sign * math.floor(at / step) * step
            d = {k: v.cuda() if torch.is_tensor(v) else v
                 for k, v in dict(s, z=(z + offset).to(act)).items()}
            assert torch.equal(d["z"].cpu().double() - offset, z)
            loss, grad = _lm().distill(tau=tau, kd_weight=0.7, ce_weight=ce, **d)
            # (the offset changes nothing)
            want_l, want_g, el, eg = _reference(dict(s, z=z), tau, 0.7, ce)
            acc = F64 if act == F64 else F32
            _within(loss, want_l, el, acc, acc)
            _within(grad, want_g, eg, acc, act)


def test_small_temperatures():
    """A temperature that makes z / tau large: the largest logits share the
    probability."""
    lm = _lm()
    announce("distill, small temperatures")
    for V in (200, 30000):
        for act in (BF16, F32, F64):
            z = torch.full((2, V), -3.0, dtype=act, device="cuda")
            z[0, 5] = z[0, V - 7] = 9.0
            z[1, 11] = -0.75
            top = torch.tensor([[3.0, 3.0, 1.0], [-9.0, -11.0, -9.0]], device="cuda")
            idx = torch.tensor([[5, V - 7, 2], [11, 0, 1]], dtype=torch.int32, device="cuda")
            for tau in (1e-4, 1e-6, 1e-10, 1e-15):
                loss, grad = lm.distill(z, top, idx, tau)
                grad = grad.double() / tau
                assert torch.isfinite(loss[0]) and loss[0].abs() <= 1e-6 * tau * tau
                assert grad[0].abs().max() <= 1e-6
                want = torch.zeros(V, dtype=F64, device="cuda")
                want[11], want[1] = 0.5, -0.5
                assert (grad[1] - want).abs().max() <= 2.0 ** -8


def test_work_buffers_that_do_not_hold():
    """Work buffers on the host, too small, or with fewer elements in memory than
    they show are refused, as are operands apart from each other."""
    lm = _lm()
    announce("distill, work buffers")
    z, top = torch.zeros((2, 9000), device="cuda"), torch.zeros((2, 3), device="cuda")
    idx = torch.zeros((2, 3), dtype=torch.int32, device="cuda")

    def call(work):
        return lm.distill(z, top, idx, work=work)
    size = 1 << 24
    for work in (torch.empty(size, dtype=torch.uint8), torch.empty(8, device="cuda")[:1],
                 torch.empty(1, dtype=torch.uint8, device="cuda").expand(size),
                 torch.empty(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            call(work)
    call(torch.empty(size, dtype=torch.uint8, device="cuda"))


def test_gradient_beside_the_logits():
    """Logits and gradient as columns of one buffer."""
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("distill, gradient beside the logits")
    N, V = 5, 301
    d = {k: v.cuda() for k, v in _inputs(N, V, 7, BF16).items()}
    want = lm.distill(ce_weight=0.3, **d)
    wide = torch.full((N, 2 * V + 1), 5.0, dtype=BF16, device="cuda")
    wide[:, :V] = d["z"]
    d["z"] = wide[:, :V]
    got = lm.distill(ce_weight=0.3, grad=wide[:, V:2 * V], **d)
    assert torch.equal(got[0], want[0]) and torch.equal(wide[:, V:2 * V], want[1])
    assert (wide[:, 2 * V] == 5).all()
    for k in (V - 1, 1):
        with pytest.raises(E.EccError) as e:
            lm.distill(grad=wide[:, k:k + V], **d)
        assert e.value.status == E.ECC_ERR_ARG


@pytest.mark.parametrize("act,V,K,in_place", [(BF16, 3, 2, False), (F32, 2, 0, True)])
def test_more_rows_than_one_launch_takes(act, V, K, in_place):
    """Rows of more than 2^32 threads: all repeats of some rows give the same."""
    lm = _lm()
    N = 2 * (1 << 31) // 64 + 1003      # (64 threads to a row)
    announce("distill, many launches", act, N, V, K)
    n = 997
    s = {k: v.cuda() for k, v in _inputs(n, V, K, act, absent=0.1).items()}
    d = {k: v.repeat(-(-N // n), *[1] * (v.dim() - 1))[:N] for k, v in s.items()}
    want = lm.distill(tau=2.0, kd_weight=0.7, ce_weight=0.3, **s)
    loss, grad = lm.distill(tau=2.0, kd_weight=0.7, ce_weight=0.3,
                            grad=d["z"] if in_place else True, **d)
    for got, w in ((loss, want[0]), (grad, want[1])):
        whole = N // n * n
        step = n * 4096
        for at in range(0, whole, step):
            hi = min(whole, at + step)
            assert (got[at:hi].view(-1, n, *w.shape[1:]) == w).all()
        assert torch.equal(got[whole:], w[:N - whole])
