"""The norms, gate and residual around a block through the library's calls,
forward and backward, against their definitions in 64 bits.

Tolerances.  With u the unit roundoff of the sums (2^-24, 2^-53 in fp64) and
r that of the stored result (2^-8 for bf16), a row's sum of up to 16,384
squares is added by threads of up to 16 elements, lanes and waves: fewer than
40 additions in a chain, so a norm factor is within 40 u (48 u with its root
and quotient) of its value.  Everything else is a few products and sums:
60 u of the sum of the terms' magnitudes bounds a forward result.  The
gradients' two corrections repeat this with sums of their own: 100 u of the
magnitudes for dX, 200 u for df; a sum over m rows adds m u more."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from gpu_common import announce                           # noqa: E402

pytestmark = pytest.mark.gpu

F64, F32, BF16 = torch.float64, torch.float32, torch.bfloat16
ULP = {F64: 2.0 ** -53, F32: 2.0 ** -24, BF16: 2.0 ** -8}
EPS = 1e-5


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


def _random(shape, dtype, seed, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g, dtype=F64) * scale + shift).to(dtype)


def _inputs(N, D, act, wt, gate="none", gate_rows=1, post=True, pre=True, seed=0):
    s = dict(x=_random((N, D), act, seed + 1, 2.0), f=_random((N, D), act, seed + 2, 0.7),
             w_post=_random((D,), wt, seed + 3, 0.2, 1.0) if post else None,
             w_pre=_random((D,), wt, seed + 4, 0.2, 1.0) if pre else None, gate=None,
             gate_rows=gate_rows)
    if gate == "rows":
        s["gate"] = _random((-(-N // gate_rows), D), act, seed + 5, 0.5, 0.5)
    elif gate == "param":
        s["gate"], s["gate_rows"] = _random((D,), wt, seed + 5, 0.5, 0.5), 0
    return s


def _gpu_args(s):
    return {k: v.cuda() if torch.is_tensor(v) else v for k, v in s.items()}


def _gate_of_rows(s, N):
    g = s["gate"]
    if g is None:
        return torch.ones((N, 1), dtype=F64)
    if s["gate_rows"] == 0:
        return g.double().expand(N, -1)
    return g.double()[torch.arange(N) // s["gate_rows"]]


def _forward_ref(s, a, b, o):
    """x', h and bounds of their errors in units of u."""
    x = s["x"].double()
    N = x.shape[0]
    y, ex = a * x, 8 * (a * x).abs()
    if s["f"] is not None:
        f = s["f"].double()
        branch = f
        if s["w_post"] is not None:
            branch = f * torch.rsqrt((f * f).mean(1, keepdim=True) + EPS) * \
                (o + s["w_post"].double())
        branch = b * _gate_of_rows(s, N) * branch
        y, ex = y + branch, ex + 60 * branch.abs()
    if s["w_pre"] is None:
        return y, ex, None, None
    q = torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
    w = o + s["w_pre"].double()
    h = y * q * w
    spread = torch.linalg.norm(ex, dim=1, keepdim=True) / \
        torch.linalg.norm(y, dim=1, keepdim=True).clamp_min(1e-300)
    return y, ex, h, (q * w).abs() * ex + h.abs() * (60 + spread)


def _within(got, want, bound_u, acc, out_type):
    got = got.cpu().double()
    u = 2.0 ** -53 if acc == F64 else 2.0 ** -24
    tol = bound_u * u + ULP[out_type] * (want.abs() + bound_u * u)
    bad = (got - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), float(((got - want).abs() / tol.clamp_min(1e-300)).max()))


def _check_forward(s, a=1.0, b=1.0, o=0.0):
    act = s["x"].dtype
    x, h = _lm().norm_forward(res_scale=a, branch_scale=b, eps=EPS, offset=o, **_gpu_args(s))
    y, ey, r, er = _forward_ref(s, a, b, o)
    if x is not None:
        _within(x, y, ey, act, act)
    if r is None:
        assert h is None
    else:
        _within(h, r, er, act, act)


SIZES = [(1, 1), (1, 2), (3, 7), (5, 64), (2, 511), (4, 1000), (3, 1025), (2, 2050), (3, 4096),
         (2, 5001), (1, 8192)]


@pytest.mark.parametrize("act,wt", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16),
                                    (F64, F64), (F64, F32)])
@pytest.mark.parametrize("N,D", SIZES)
def test_forward(act, wt, N, D):
    announce("norm", act, wt, N, D)
    for gate in ("none", "rows", "param"):
        _check_forward(_inputs(N, D, act, wt, gate), 0.9, 0.7, 0.0)
    _check_forward(_inputs(N, D, act, wt, pre=False), 1.0, 1.0, 1.0)
    _check_forward(_inputs(N, D, act, wt, "rows", post=False), 1.1, -0.5, 0.0)
    s = _inputs(N, D, act, wt, post=False)
    s["f"] = None
    _check_forward(s, 1.0, 1.0, 1.0)
    _check_forward(s, 0.5, 1.0, 0.0)


@pytest.mark.parametrize("act,D", [(BF16, 12001), (BF16, 16384), (F32, 16384), (F32, 9000)])
def test_forward_longest_rows(act, D):
    announce("norm, longest rows", act, D)
    _check_forward(_inputs(3, D, act, F32, "rows"), 0.9, 0.7)


@pytest.mark.parametrize("N,g", [(700, 1), (700, 7), (700, 256), (701, 100), (5000, 5000),
                                 (4099, 64)])
def test_forward_many_rows(N, g):
    """More rows than workgroups; gates shared by runs of rows, the last run
    short."""
    announce("norm, many rows", N, g)
    _check_forward(_inputs(N, 96, BF16, F32, "rows", gate_rows=g))
    _check_forward(_inputs(N, 2048, BF16, F32, "rows", gate_rows=g))


def test_forward_no_rows():
    lm = _lm()
    announce("norm, no rows")
    x = torch.empty((0, 40), device="cuda")
    w = torch.ones(40, device="cuda")
    y, h = lm.norm_forward(x, x.clone(), w_post=w, w_pre=w)
    assert y.shape == h.shape == (0, 40)


def test_forward_zero_and_extreme_rows():
    """Rows of zeros give zeros; large and small rows keep their norm; NaN and
    infinity stay in their row."""
    lm = _lm()
    announce("norm, extreme rows")
    x = torch.zeros((6, 300), dtype=F32)
    x[1], x[2], x[3, 5], x[4, 7] = 1e15, 1e-15, float("nan"), float("inf")
    x[5] = 3.0
    w = torch.ones(300)
    _, h = lm.norm_forward(x.cuda(), w_pre=w.cuda(), eps=1e-30)
    h = h.cpu()
    assert (h[0] == 0).all() and torch.isnan(h[3]).all() and torch.isnan(h[4, 7])
    for r in (1, 5):
        assert torch.allclose(h[r], torch.ones(300), rtol=1e-5)
    assert torch.allclose(h[2], torch.full((300,), 1e-15 / (2e-30 ** 0.5)), rtol=1e-5)


def test_forward_strides_and_places():
    """Operands as views of wider buffers, results in place of operands."""
    lm = _lm()
    announce("norm, strides")
    N, D = 37, 205
    s = _inputs(N, D, BF16, F32, "rows", gate_rows=4)
    wide = {k: torch.full((s[k].shape[0], D + 3 + i), 7.0, dtype=BF16, device="cuda")
            for i, k in enumerate(("x", "f", "gate"))}
    view = {k: w[:, 1 + i:1 + i + D] for i, (k, w) in enumerate(wide.items())}
    for k in view:
        view[k].copy_(s[k])
    kw = dict(w_post=s["w_post"].cuda(), w_pre=s["w_pre"].cuda(), gate=view["gate"], gate_rows=4)
    want = lm.norm_forward(**_gpu_args(s))
    got = lm.norm_forward(view["x"], view["f"], **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    lm.norm_forward(view["x"], view["f"], x_out=view["x"], h=view["f"], **kw)
    assert torch.equal(view["x"], want[0]) and torch.equal(view["f"], want[1])
    assert (wide["x"][:, 0] == 7).all() and (wide["x"][:, 1 + D:] == 7).all()
    assert (wide["f"][:, :2] == 7).all() and (wide["f"][:, 2 + D:] == 7).all()
    # rows of a batch of sequences
    x3 = s["x"][:36].view(4, 9, D).cuda()
    y, _ = lm.norm_forward(x3, x3.clone())
    assert y.shape == x3.shape


# ---------------------------------------------------------------------------
# backward
# ---------------------------------------------------------------------------

def _grad_ref(s, dh, dxo, a, b, o, P):
    """Gradients and bounds of their errors in units of u."""
    x = s["x"].double()
    N, D = x.shape
    zero = torch.zeros((N, D), dtype=F64)
    d = zero if dxo is None else dxo.double()
    md = d.abs()
    out, err = {}, {}
    rows = N // P

    def per_worker(t):
        return t.view(P, rows, D).sum(1)

    if s["w_pre"] is not None:
        q = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
        A = dh.double() * (o + s["w_pre"].double())
        d = d + q * (A - x * q * q * (A * x).mean(1, keepdim=True))
        md = md + q * (A.abs() + x.abs() * q * q * (A * x).abs().mean(1, keepdim=True))
        t = dh.double() * x * q
        out["dw_pre"], err["dw_pre"] = per_worker(t), (rows + 100) * per_worker(t.abs())
    out["dx"], err["dx"] = a * d, 100 * abs(a) * md
    if s["f"] is None:
        return out, err
    f = s["f"].double()
    g = _gate_of_rows(s, N)
    w = o + s["w_post"].double() if s["w_post"] is not None else 1.0
    k = torch.rsqrt((f * f).mean(1, keepdim=True) + EPS) if s["w_post"] is not None else 1.0
    u = f * k * w
    if s["gate"] is not None:
        t, m = b * d * u, abs(b) * md * u.abs()
        if s["gate_rows"] == 0:
            out["dgate"], err["dgate"] = per_worker(t), (rows + 200) * per_worker(m)
        else:
            at = torch.arange(N) // s["gate_rows"]
            n = s["gate"].shape[0]
            out["dgate"] = torch.zeros((n, D), dtype=F64).index_add_(0, at, t)
            err["dgate"] = torch.zeros((n, D), dtype=F64).index_add_(0, at, m) * \
                (s["gate_rows"] + 200)
    du, mdu = b * g * d, abs(b) * g.abs() * md
    if s["w_post"] is not None:
        t = du * f * k
        out["dw_post"] = per_worker(t)
        err["dw_post"] = (rows + 200) * per_worker(mdu * f.abs() * k)
        B, mB = du * w, mdu * w.abs()
        out["df"] = k * (B - f * k * k * (B * f).mean(1, keepdim=True))
        err["df"] = 200 * k * (mB + f.abs() * k * k * (mB * f.abs()).mean(1, keepdim=True))
    else:
        out["df"], err["df"] = du, 200 * mdu
    return out, err


def _check_grad(s, a=1.0, b=1.0, o=0.0, P=1, gt=None, with_dxo=True, seed=50):
    act = s["x"].dtype
    N, D = s["x"].shape
    dh = _random((N, D), act, seed, 0.3) if s["w_pre"] is not None else None
    dxo = _random((N, D), act, seed + 1, 0.3) if with_dxo else None
    wt = next((s[k].dtype for k in ("w_post", "w_pre") if s[k] is not None), act)
    gt = gt or (s["gate"].dtype if s["gate"] is not None and s["gate_rows"] == 0 else wt)
    kw = dict(_gpu_args(s), dh=None if dh is None else dh.cuda(),
              dx_out=None if dxo is None else dxo.cuda(), res_scale=a, branch_scale=b, eps=EPS,
              offset=o, P=P, dtype=gt)
    got = _lm().norm_grad(**kw)
    want, err = _grad_ref(s, dh, dxo, a, b, o, P)
    assert {k for k, v in got.items() if v is not None} == set(want)
    for k in want:
        rows = k in ("dx", "df") or (k == "dgate" and s["gate_rows"])
        _within(got[k], want[k], err[k], act, act if rows else gt)
    again = _lm().norm_grad(**kw)
    assert all(torch.equal(got[k], again[k]) for k in want)
    return got


@pytest.mark.parametrize("act,wt", [(BF16, BF16), (BF16, F32), (F32, F32), (F64, F64)])
@pytest.mark.parametrize("N,D", SIZES + [(40, 33)])
def test_grad(act, wt, N, D):
    announce("norm grad", act, wt, N, D)
    for gate in ("none", "rows", "param"):
        _check_grad(_inputs(N, D, act, wt, gate), 0.9, 0.7, 0.0)
    _check_grad(_inputs(N, D, act, wt, pre=False), 1.0, 1.0, 1.0)
    _check_grad(_inputs(N, D, act, wt, "rows", post=False), 1.1, -0.5, 0.0)
    _check_grad(_inputs(N, D, act, wt, "param"), 1.0, 1.0, 1.0, with_dxo=False)
    s = _inputs(N, D, act, wt, post=False)
    s["f"] = None
    _check_grad(s, 0.5, 1.0, 0.0, gt=F64)


@pytest.mark.parametrize("act,D", [(BF16, 9001), (BF16, 16384), (F32, 16384)])
def test_grad_longest_rows(act, D):
    announce("norm grad, longest rows", act, D)
    _check_grad(_inputs(5, D, act, F32, "rows", gate_rows=5), 0.9, 0.7)


@pytest.mark.parametrize("D", [40, 515, 1030])
@pytest.mark.parametrize("N,P,g", [(900, 1, 1), (900, 1, 13), (901, 1, 450), (20000, 1, 20000),
                                   (9000, 3, 3000), (9000, 3, 1500), (9000, 9, 10),
                                   (9030, 6, 215), (17, 17, 1)])
def test_grad_shared_gates_and_workers(D, N, P, g):
    """Gate rows shared by runs of rows shorter and longer than a unit's, the
    last run short; workers' sums apart."""
    announce("norm grad, shared gates", D, N, P, g)
    _check_grad(_inputs(N, D, F32, F32, "rows", gate_rows=g), 0.9, 0.7, P=P)
    _check_grad(_inputs(N, D, BF16, F32, "param"), 0.9, 0.7, P=P, gt=F64)


def test_grad_accumulate_in_contributions():
    """Parameters' gradients added inside workers' contributions, in place of
    dx_out and dh where that is allowed."""
    lm = _lm()
    announce("norm grad, contributions")
    P, n, D = 3, 70, 130
    s = _inputs(P * n, D, F32, F32, "param")
    base = _random((P, 3 * D + 11), F64, 60)
    contrib = base.cuda()
    views = dict(dw_post=contrib[:, 2:2 + D], dw_pre=contrib[:, 2 + D:2 + 2 * D],
                 dgate=contrib[:, 5 + 2 * D:5 + 3 * D])
    dh, dxo = _random((P * n, D), F32, 61), _random((P * n, D), F32, 62)
    kw = dict(_gpu_args(s), P=P, eps=EPS)
    want = lm.norm_grad(dh=dh.cuda(), dx_out=dxo.cuda(), dtype=F64, **kw)
    d_h, d_o = dh.cuda(), dxo.cuda()
    got = lm.norm_grad(dh=d_h, dx_out=d_o, dx=d_o, df=d_h, accumulate=True, **views, **kw)
    assert torch.equal(d_o, want["dx"]) and torch.equal(d_h, want["df"])
    assert got["dx"] is d_o
    expect = base.cuda()
    for k, at in (("dw_post", 2), ("dw_pre", 2 + D), ("dgate", 5 + 2 * D)):
        expect[:, at:at + D] += want[k]
    assert torch.equal(contrib, expect)


def test_grad_zero_rows():
    """Rows of zeros, with an eps whose norm factor has a cube beyond fp32: the
    gradient is the incoming one times the weight and the factor."""
    lm = _lm()
    announce("norm grad, zero rows")
    x = torch.zeros((4, 50), device="cuda")
    x[2] = 1.0
    w = torch.full((50,), 2.0, device="cuda")
    dh = torch.full((4, 50), 3.0, device="cuda")
    g = lm.norm_grad(x, x.clone(), dh, None, w_post=w, w_pre=w, eps=1e-30)
    assert torch.isfinite(g["dx"]).all()
    assert torch.allclose(g["dx"][[0, 1, 3]], torch.full((3, 50), 6e15, device="cuda"), rtol=1e-5)
    assert torch.isfinite(g["dw_pre"]).all() and torch.isfinite(g["dw_post"]).all()


@pytest.mark.parametrize("act,D", [(BF16, 8192), (BF16, 10000), (F64, 3000)])
def test_grad_wide_rows_in_a_graph(act, D):
    """Shapes whose weights fill more LDS than a kernel has by default, and those
    that keep none there, captured and replayed."""
    lm = _lm()
    announce("norm grad, wide rows in a graph", act, D)
    s = _gpu_args(_inputs(40, D, act, F32 if act != F64 else F64, "rows", gate_rows=8))
    dh, dxo = _random((40, D), act, 90).cuda(), _random((40, D), act, 91).cuda()
    lm.norm_grad(**s, dh=dh, dx_out=dxo)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lm.norm_grad(**s, dh=dh, dx_out=dxo)
    for k in range(3):
        s["x"].copy_(_random((40, D), act, 95 + k))
        graph.replay()
        torch.cuda.synchronize()
        want = lm.norm_grad(**s, dh=dh, dx_out=dxo)
        assert all(torch.equal(got[k], want[k]) for k in want)


def test_grad_no_rows():
    lm = _lm()
    announce("norm grad, no rows")
    x = torch.empty((0, 40), device="cuda")
    w = torch.ones(40, device="cuda")
    g = lm.norm_grad(x, x.clone(), x.clone(), w_post=w, w_pre=w, P=2)
    assert not g["dw_pre"].any() and not g["dw_post"].any() and g["dx"].shape == (0, 40)
    held = torch.full((1, 40), 3.0, device="cuda")
    lm.norm_grad(x, None, x.clone(), w_pre=w, dw_pre=held, accumulate=True)
    assert (held == 3).all()


@pytest.mark.parametrize("gate", ["none", "rows", "param"])
def test_grad_against_differences(gate):
    """Central differences of sum(c_x x' + c_h h) along random directions, the
    forward calls in 64 bits (step t: error of the order t^2)."""
    lm = _lm()
    announce("norm grad, differences", gate)
    N, D, a, b = 6, 30, 0.8, 0.6
    s = _inputs(N, D, F64, F64, gate, gate_rows=2)
    cx, ch = _random((N, D), F64, 70).cuda(), _random((N, D), F64, 71).cuda()
    kw = dict(res_scale=a, branch_scale=b, eps=EPS, offset=1.0)

    def value(t):
        x, h = lm.norm_forward(**_gpu_args(t), **kw)
        return float((cx * x).sum() + (ch * h).sum())

    x_out, _ = lm.norm_forward(**_gpu_args(s), **kw)
    g = lm.norm_grad(**_gpu_args(dict(s, x=x_out)), dh=ch, dx_out=cx, **kw)
    for k, name in (("x", "dx"), ("f", "df"), ("w_post", "dw_post"), ("w_pre", "dw_pre"),
                    ("gate", "dgate")):
        if s[k] is None:
            continue
        for j in range(3):
            v = _random(s[k].shape, F64, 80 + j)
            t = 1e-4
            up, down = dict(s, **{k: s[k] + t * v}), dict(s, **{k: s[k] - t * v})
            numeric = (value(up) - value(down)) / (2 * t)
            exact = float((g[name].cpu().reshape(s[k].shape) * v).sum())
            scale = float(g[name].abs().sum().cpu()) + 1.0
            assert abs(numeric - exact) <= 1e-6 * scale, (k, numeric, exact)


def test_on_another_stream_and_in_a_graph():
    lm = _lm()
    announce("norm, stream and graph")
    s = _gpu_args(_inputs(300, 260, BF16, F32, "rows", gate_rows=50))
    dh, dxo = _random((300, 260), BF16, 90).cuda(), _random((300, 260), BF16, 91).cuda()
    want = lm.norm_forward(**s), lm.norm_grad(**s, dh=dh, dx_out=dxo)

    def same(got):
        return torch.equal(got[0][0], want[0][0]) and torch.equal(got[0][1], want[0][1]) and \
            all(torch.equal(got[1][k], want[1][k]) for k in want[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = lm.norm_forward(**s), lm.norm_grad(**s, dh=dh, dx_out=dxo)
    torch.cuda.current_stream().wait_stream(side)
    assert same(got)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lm.norm_forward(**s), lm.norm_grad(**s, dh=dh, dx_out=dxo)
    for k in range(3):
        s["x"].copy_(_random((300, 260), BF16, 95 + k))
        graph.replay()
        torch.cuda.synchronize()
        want = lm.norm_forward(**s), lm.norm_grad(**s, dh=dh, dx_out=dxo)
        assert same(got)


def test_refusals():
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("norm refusals")
    x, f, w = (torch.zeros(s, device="cuda") for s in ((6, 8), (6, 8), (8,)))
    gate, h, o = (torch.zeros(s, device="cuda") for s in ((3, 8), (6, 8), (6, 8)))

    def desc(**kw):
        d = dict(n=3, D=8, P=2, type=E.ECC_F32, w_type=E.ECC_F32, d_x=x.data_ptr(), ld_x=8,
                 d_f=f.data_ptr(), ld_f=8, d_gate=None, ld_gate=8, gate_rows=1,
                 d_w_post=w.data_ptr(), d_w_pre=w.data_ptr(), w_offset=0.0, res_scale=1.0,
                 branch_scale=1.0, eps=1e-6)
        d.update(kw)
        return E.ecc_norm_t(**d)

    def status(call, *args):
        with pytest.raises(E.EccError) as e:
            call(*args)
        return e.value.status

    bad_desc = [dict(n=-1), dict(D=0), dict(P=0), dict(type=3), dict(w_type=-1), dict(eps=0.0),
                dict(eps=-1.0), dict(eps=float("nan")), dict(gate_rows=-1), dict(ld_x=7),
                dict(ld_f=7), dict(w_type=E.ECC_F64), dict(d_f=None),
                dict(d_gate=gate.data_ptr(), ld_gate=7), dict(d_x=x.data_ptr() + 2),
                dict(d_gate=gate.data_ptr(), gate_rows=2), dict(d_w_pre=w.data_ptr() + 1)]
    for bad in bad_desc:
        assert status(E.ecc_norm_forward, desc(**bad), o, 8, h, 8) == E.ECC_ERR_ARG, bad
        assert E.ecc_norm_work_size(desc(**bad)) == -1
    for D, t in ((16385, E.ECC_F32), (16385, E.ECC_BF16), (8193, E.ECC_F64)):
        wide = desc(D=D, type=t, ld_x=D, ld_f=D)
        assert status(E.ecc_norm_forward, wide, o, D, h, D) == E.ECC_ERR_RANGE
    for args in ((o, 8, None, 0), (None, 0, None, 0), (o, 7, h, 8), (o, 8, h, 7), (o, 8, o, 8),
                 (f, 8, h, 8), (o, 8, w, 8), (o.data_ptr() + 2, 8, h, 8)):
        assert status(E.ecc_norm_forward, desc(), *args) == E.ECC_ERR_ARG, args
    assert status(E.ecc_norm_forward, desc(d_w_pre=None), o, 8, h, 8) == E.ECC_ERR_ARG
    assert status(E.ecc_norm_forward, desc(d_x=None), o, 8, h, 8) == E.ECC_ERR_ARG

    work = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p = [torch.zeros((2, 8), device="cuda") for _ in range(2)]

    def grad(**kw):
        d = dict(d_dh=h.data_ptr(), ld_dh=8, d_dx_out=None, ld_dx_out=8, d_dx=o.data_ptr(),
                 ld_dx=8, d_df=f.data_ptr(), ld_df=8, d_dgate=None, ld_dgate=8,
                 d_dw_post=p[0].data_ptr(), d_dw_pre=p[1].data_ptr(), grad_type=E.ECC_F32,
                 accumulate=0, worker_stride=8)
        d.update(kw)
        return E.ecc_norm_grad_t(**d)

    E.ecc_norm_grad(desc(), grad(), work)
    for bad in (dict(d_dh=None), dict(grad_type=8), dict(accumulate=3), dict(ld_dh=7),
                dict(ld_dx=7), dict(ld_df=7), dict(worker_stride=7), dict(d_dgate=o.data_ptr()),
                dict(d_dx=x.data_ptr()), dict(d_dx=f.data_ptr(), d_df=None),
                dict(d_df=o.data_ptr()), dict(d_dw_pre=p[0].data_ptr()),
                dict(d_dw_pre=w.data_ptr()), dict(d_dx=h.data_ptr(), d_df=h.data_ptr()),
                dict(d_dx=None, d_df=None, d_dw_post=None, d_dw_pre=None),
                dict(d_dx=work.data_ptr()), dict(d_dx=o.data_ptr() + 2)):
        assert status(E.ecc_norm_grad, desc(), grad(**bad), work) == E.ECC_ERR_ARG, bad
    assert status(E.ecc_norm_grad, desc(), grad(), None) == E.ECC_ERR_ARG
    assert status(E.ecc_norm_grad, desc(), grad(), work.data_ptr() + 4) == E.ECC_ERR_ARG
    assert status(E.ecc_norm_grad, desc(d_w_post=None), grad(), work) == E.ECC_ERR_ARG
    # what the tensors say
    for kw in (dict(f=f[:5]), dict(f=f.double()), dict(f=f, gate=gate[:2], gate_rows=2),
               dict(f=f, w_post=w[:7]), dict(f=f, w_post=w, w_pre=w.double()),
               dict(f=f.t().contiguous().t()), dict(f=f, h=h)):
        with pytest.raises(ValueError):
            lm.norm_forward(x, **kw)
    with pytest.raises(TypeError):
        lm.norm_forward(x.half(), f.half())
    with pytest.raises(ValueError):
        lm.norm_grad(x, f, h, w_pre=w, P=4)
    with pytest.raises(ValueError):
        lm.norm_grad(x, f, h, w_pre=w, accumulate=True)


def _strictly_within(got, want, bound_u, acc, out_type):
    """_within, for which a NaN of either side is a difference too."""
    assert torch.isfinite(want).all() and torch.isfinite(got).all()
    _within(got, want, bound_u, acc, out_type)


@pytest.mark.parametrize("act,D", [(F64, 3000), (F64, 4096), (BF16, 9001), (BF16, 16384),
                                   (F32, 9001)])
@pytest.mark.parametrize("N,g", [(8, 5), (1000, 900), (1000, 300)])
def test_grad_long_rows_short_last_gate(act, D, N, g):
    """Rows that are not held, in groups split over units, the last group short:
    units without rows add nothing, whatever the work buffer held."""
    announce("norm grad, long rows, short last gate", act, D, N, g)
    wt = F64 if act == F64 else F32
    s = _inputs(N, D, act, wt, "rows", gate_rows=g)
    dh, dxo = _random((N, D), act, 50, 0.3), _random((N, D), act, 51, 0.3)
    work = torch.full((3 * 1024 * D * 8,), 255, dtype=torch.uint8, device="cuda")
    got = _lm().norm_grad(**_gpu_args(s), dh=dh.cuda(), dx_out=dxo.cuda(), res_scale=0.9,
                          branch_scale=0.7, eps=EPS, work=work)
    want, err = _grad_ref(s, dh, dxo, 0.9, 0.7, 0.0, 1)
    for k in want:
        out = act if k in ("dx", "df", "dgate") else wt
        _strictly_within(got[k], want[k], err[k], act, out)


@pytest.mark.parametrize("act", [BF16, F32])
@pytest.mark.parametrize("N,P,D", [(40000, 1, 64), (40000, 4, 128), (9000, 3, 512), (6000, 2, 1024),
                                   (3000, 1, 4096), (2001, 3, 8192), (1000, 2, 16384), (1, 1, 8)])
def test_grad_fp64_sums_over_rows(act, N, P, D):
    """fp64 gradients of fp32 and bf16 rows are sums in fp64.  Rows of one
    magnitude, weights and scales are powers of two, so that norm factors and
    every row's term are exact: m additions in fp64 are within (m + 4) 2^-53 of
    the magnitudes' sum."""
    lm = _lm()
    announce("norm grad, fp64 sums", act, N, P, D)
    g = torch.Generator(device="cuda").manual_seed(N + D)

    def signs(scale):
        return ((torch.randint(0, 2, (N, D), generator=g, device="cuda") * 2 - 1) * scale).to(act)

    x, f = signs(2.0), signs(4.0)
    dh, dxo = (torch.randn((N, D), generator=g, device="cuda").to(act) for _ in range(2))
    one = torch.ones(D, device="cuda")
    kw = dict(eps=1e-30, P=P, dtype=F64)

    def check(got, terms):
        t = terms.view(P, N // P, D)
        assert got.dtype == F64
        assert ((got - t.sum(1)).abs() <= (N // P + 4) * 2.0 ** -53 * t.abs().sum(1)).all()

    got = lm.norm_grad(x, None, dh, dxo, w_pre=one, **kw)
    check(got["dw_pre"], dh.double() * x.double() / 2)
    got = lm.norm_grad(x, f, None, dxo, w_post=2 * one, gate=one / 4, gate_rows=0,
                       branch_scale=0.5, **kw)
    check(got["dw_post"], dxo.double() * f.double() / 4 / 8)
    check(got["dgate"], dxo.double() * f.double() / 4)
    # beside a gate of rows, in groups longer than a unit, the last one short
    rows = 700 if P == 1 else N // P
    gate = torch.full((-(-N // rows), D), 0.25, dtype=act, device="cuda")
    got = lm.norm_grad(x, f, None, dxo, w_post=2 * one, gate=gate, gate_rows=rows,
                       branch_scale=0.5, **kw)
    check(got["dw_post"], dxo.double() * f.double() / 4 / 8)


@pytest.mark.parametrize("act", [BF16, F32])
def test_eps_below_fp32(act):
    """An eps that fp32 rounds to zero: rows of zeros still give zeros."""
    lm = _lm()
    announce("norm, tiny eps", act)
    x = torch.zeros((3, 70), dtype=act, device="cuda")
    x[1] = 2.0
    w = torch.ones(70, device="cuda")
    for eps in (1e-50, 1e-300, 5e-324):
        y, h = lm.norm_forward(x, x.clone(), w_post=w, w_pre=w, eps=eps)
        assert not y[[0, 2]].any() and not h[[0, 2]].any()
        assert torch.allclose(h[1].float(), torch.ones(70, device="cuda"), rtol=1e-2)
        g = lm.norm_grad(x, x.clone(), torch.zeros_like(x), None, w_post=w, w_pre=w, eps=eps)
        assert all(not g[k].any() for k in ("dx", "df", "dw_post", "dw_pre"))


def test_work_buffers_that_do_not_hold():
    """Work buffers on the host, too small, or with fewer elements in memory than
    they show are refused, as are operands apart from each other."""
    lm = _lm()
    announce("norm, work buffers")
    x, w = torch.zeros((6, 8), device="cuda"), torch.ones(8, device="cuda")

    def call(work):
        return lm.norm_grad(x, None, x.clone(), w_pre=w, work=work)
    size = 1 << 24
    for work in (torch.empty(size, dtype=torch.uint8), torch.empty(8, device="cuda")[:1],
                 torch.empty(1, dtype=torch.uint8, device="cuda").expand(size),
                 torch.empty(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            call(work)
    call(torch.empty(size, dtype=torch.uint8, device="cuda"))


def test_workers_gradients_that_overlap():
    """A parameter's gradient of one worker in the place of another parameter's
    of the next worker is refused; one beside the other is not."""
    from paper_2203_17063_amd import capi as E
    announce("norm grad, workers' overlap")
    P, n, D = 3, 4, 16
    s = _gpu_args(_inputs(P * n, D, F32, F32))
    dh = torch.zeros((P * n, D), device="cuda")
    flat = torch.zeros(4096, device="cuda")

    def at(first, stride=64):
        return torch.as_strided(flat, (P, D), (stride, 1), first)

    for first in (64, 128, 64 + 15, 64 - 15, 128 + 3):
        with pytest.raises(E.EccError) as e:
            _lm().norm_grad(dh=dh, P=P, dw_post=at(0), dw_pre=at(first), **s)
        assert e.value.status == E.ECC_ERR_ARG
    for first in (16, 48, 64 + 16, 64 + 48, 192, 192 + 5):
        _lm().norm_grad(dh=dh, P=P, dw_post=at(0), dw_pre=at(first), **s)


def test_rows_beside_each_other():
    """Operands and results as columns of one buffer, which share no element; by
    one column less they do, and are refused."""
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("norm, rows beside each other")
    N, D = 9, 37
    s = _gpu_args(_inputs(N, D, F32, F32))
    dh, dxo = _random((N, D), F32, 61).cuda(), _random((N, D), F32, 62).cuda()
    want, want_g = lm.norm_forward(**s), lm.norm_grad(dh=dh, dx_out=dxo, **s)
    wide = torch.full((N, 4 * D + 2), 5.0, device="cuda")
    x, f, y, h = (wide[:, 1 + k * D:1 + (k + 1) * D] for k in range(4))
    x.copy_(s["x"])
    f.copy_(s["f"])
    t = dict(s, x=x, f=f)
    lm.norm_forward(x_out=y, h=h, **t)
    assert torch.equal(y, want[0]) and torch.equal(h, want[1]) and torch.equal(x, s["x"])
    lm.norm_grad(dh=dh, dx_out=dxo, dx=h, df=y, **t)
    assert torch.equal(h, want_g["dx"]) and torch.equal(y, want_g["df"])
    assert (wide[:, 0] == 5).all() and (wide[:, -1] == 5).all()
    for k in (1 + 2 * D - 1, D + 2, 2 * D, 3):
        with pytest.raises(E.EccError) as e:
            lm.norm_forward(x_out=wide[:, k:k + D], h=h, **t)
        assert e.value.status == E.ECC_ERR_ARG


def test_grad_given_beside_new():
    """One parameter's gradient given as a view of wide contributions: the
    others take no more memory than they hold."""
    lm = _lm()
    announce("norm grad, one given")
    P, n, D, m = 8, 20, 64, 1 << 22
    s = _gpu_args(_inputs(P * n, D, F32, F32, "param"))
    dh, dxo = _random((P * n, D), F32, 61).cuda(), _random((P * n, D), F32, 62).cuda()
    want = lm.norm_grad(dh=dh, dx_out=dxo, P=P, **s)
    contrib = torch.full((P, m), 3.0, device="cuda")
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    got = lm.norm_grad(dh=dh, dx_out=dxo, P=P, dw_pre=contrib[:, 5:5 + D], **s)
    assert torch.cuda.max_memory_allocated() - before < P * m
    for k in want:
        assert torch.equal(got[k], want[k]), k
    assert got["dw_pre"].data_ptr() == contrib[:, 5:].data_ptr()
    contrib[:, 5:5 + D] = 3.0
    assert (contrib == 3).all()
    got = lm.norm_grad(dh=dh, dx_out=dxo, P=P, dw_pre=contrib[:, 5:5 + D],
                       dgate=contrib[:, 5 + D:5 + 2 * D], **s)
    assert all(torch.equal(got[k], want[k]) for k in want)
    for at in (5 + D - 1, 6, 4):
        with pytest.raises(ValueError):
            lm.norm_grad(dh=dh, dx_out=dxo, P=P, dw_pre=contrib[:, 5:5 + D],
                         dgate=contrib[:, at:at + D], **s)


def test_grad_refusal_says_why():
    from paper_2203_17063_amd import capi as E
    announce("norm grad, refusal")
    x, w = torch.zeros((4, 8), device="cuda"), torch.ones(8, device="cuda")
    with pytest.raises(E.EccError) as e:
        _lm().norm_grad(x, None, x.clone(), w_pre=w, eps=0.0)
    assert e.value.status == E.ECC_ERR_ARG and "eps" in str(e.value)


def test_grad_of_many_workers():
    """A row each of 70,000 workers: more workgroups in the join than one launch
    of fewer than 2^32 threads has.  A worker's gradient is its row's term,
    within 100 u."""
    announce("norm grad, many workers")
    P, D = 70000, 4096
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((P, D), generator=g, device="cuda").to(BF16)
    dh = torch.randn((P, D), generator=g, device="cuda").to(BF16)
    got = _lm().norm_grad(x, None, dh, None, w_pre=torch.ones(D, device="cuda"), eps=EPS,
                          P=P)["dw_pre"]
    for lo in range(0, P, 10000):
        v = x[lo:lo + 10000].double()
        want = dh[lo:lo + 10000].double() * v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
        assert ((got[lo:lo + 10000] - want).abs() <= 101 * 2.0 ** -24 * want.abs()).all()


def test_forward_is_finite():
    """No NaN or infinity where the inputs have none (a comparison with a bound
    lets NaN pass)."""
    lm = _lm()
    announce("norm, finite")
    for act, wt in ((BF16, BF16), (BF16, F32), (F32, F32), (F64, F64)):
        for N, D in SIZES + [(3, 12001), (3, 16384), (4099, 96)]:
            if act == F64 and D > 8192:
                continue
            for gate in ("none", "rows", "param"):
                for post, pre in ((True, True), (True, False), (False, True)):
                    s = _gpu_args(_inputs(N, D, act, wt, gate, 2, post, pre))
                    for v in lm.norm_forward(res_scale=0.9, branch_scale=0.7, eps=EPS, **s):
                        assert v is None or torch.isfinite(v).all(), (act, wt, N, D, gate)


def test_workers_gradients_in_one_place():
    """A gradient whose workers share memory is refused, alone and beside one
    that was not given."""
    from paper_2203_17063_amd import capi as E
    announce("norm grad, workers in one place")
    P, D = 3, 16
    s = _gpu_args(_inputs(P * 4, D, F32, F32))
    dh, flat = torch.zeros((P * 4, D), device="cuda"), torch.zeros(4096, device="cuda")
    for stride in (0, 1, D - 1):
        t = torch.as_strided(flat, (P, D), (stride, 1))
        with pytest.raises(ValueError):
            _lm().norm_grad(dh=dh, P=P, dw_post=t, **s)
        with pytest.raises(E.EccError) as e:
            _lm().norm_grad(dh=dh, P=P, dw_post=t, dw_pre=torch.as_strided(flat, (P, D),
                                                                          (stride, 1), 512), **s)
        assert e.value.status == E.ECC_ERR_ARG
