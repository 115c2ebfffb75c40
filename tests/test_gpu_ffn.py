"""The gated feed-forward block through the library's calls, forward and
backward, against the definition in 64 bits.

Tolerances (u = 2^-24; products as in product_bounds.py).  With g and u_ off by
eg and eu, act(g) is off by at most 1.13 eg (the largest slope of either
activation) and its own arithmetic, 16 u (|g| + 1) (an exponential or error
function within 4 u, and some operations; the functions are at most |g|; bf16's
exponential of x within (1.2 |x| + 1) u, which g q (1 - q) and g^3 exp(-g^2 / 2)
make less than 4 u of); its slope by 1.2 eg (the largest second derivative is below 1.2) and 24 u.  A product
of three such factors adds 4 u.  dg and du are stored with half a step of bf16
where a gradient is bf16, or as three pieces (none)."""
import math

import pytest

torch = pytest.importorskip("torch")

from gpu_common import announce                                        # noqa: E402
from product_bounds import (BF16, F32, F64, U, ULP, product, product_error,     # noqa: E402
                            within)

pytestmark = pytest.mark.gpu


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


def _inputs(N, D, F, dtype, seed=0):
    g = torch.Generator().manual_seed(1000 * seed + N + 3 * D + 7 * F)

    def normal(shape, scale):
        return (torch.randn(shape, generator=g, dtype=F64) * scale).to(dtype).cuda()
    return (normal((N, D), 1.0), normal((F, D), 2.0 / math.sqrt(D)),
            normal((F, D), 1.0 / math.sqrt(D)), normal((N, F), 0.3))


def _act(kind, g):
    if kind == "silu":
        q = torch.sigmoid(g)
        return g * q, q * (1 + g * (1 - q))
    c = 0.5 * torch.erfc(-g * math.sqrt(0.5))
    return g * c, c + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


def _projections(x, wg, wu, act):
    """act(g), its slope, u, and bounds of their errors."""
    t = x.dtype
    g, eg = product(x.double(), wg.double().t(), t)
    u, eu = product(x.double(), wu.double().t(), t)
    a, da = _act(act, g)
    return a, 1.13 * eg + 16 * U * (g.abs() + 1), da, 1.2 * eg + 24 * U * (1 + g.abs()), u, eu


def _forward(x, wg, wu, act):
    a, ea, _, _, u, eu = _projections(x, wg, wu, act)
    return a * u, ea * (u.abs() + eu) + a.abs() * eu + 4 * U * (a * u).abs()


def _backward(x, wg, wu, dy, act, P, grad):
    """dx, dw_gate, dw_up and the bounds of their errors."""
    t = x.dtype
    a, ea, da, eda, u, eu = _projections(x, wg, wu, act)
    dy, x, wg, wu = dy.double(), x.double(), wg.double(), wu.double()
    dg, du = dy * u * da, dy * a
    edg = dy.abs() * (eu * (da.abs() + eda) + u.abs() * eda) + 4 * U * dg.abs()
    edu = dy.abs() * ea + 4 * U * du.abs()

    def stored(d, e, out):
        return e + (ULP[BF16] * (d.abs() + e) if t == BF16 and out == BF16 else 0.0)
    both = torch.cat([dg, du], 1)
    dx = product(both, torch.cat([wg, wu], 0), t,
                 torch.cat([stored(dg, edg, t), stored(du, edu, t)], 1), extra=64)
    n = x.shape[0] // P
    # (dg and du as three pieces beside x of one are three products)
    kind = F32 if grad == F32 else t

    def of_weights(d, e):
        got = [product(d[r].t(), x[r], kind, e[r].t())
               for r in (slice(p * n, (p + 1) * n) for p in range(P))]
        return tuple(torch.stack(v) for v in zip(*got))
    return dx, of_weights(dg, stored(dg, edg, grad)), of_weights(du, stored(du, edu, grad))


SIZES = [(1, 1, 1, 1), (1, 3, 7, 5), (1, 17, 64, 64), (2, 33, 65, 127), (3, 64, 128, 130),
         (5, 13, 250, 300), (1, 129, 63, 257), (4, 100, 200, 64), (1, 300, 1001, 40)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("P,n,D,F", SIZES)
def test_small(dtype, act, P, n, D, F):
    announce("ffn", dtype, act, P, n, D, F)
    x, wg, wu, dy = _inputs(P * n, D, F, dtype)
    y = _lm().gated_ffn(x, wg, wu, act=act)
    within(y, *_forward(x, wg, wu, act), "y")
    assert torch.equal(y, _lm().gated_ffn(x, wg, wu, act=act))
    for grad in {dtype, F32}:
        got = _lm().gated_ffn_grad(x, wg, wu, dy, act=act, P=P, dtype=grad)
        assert got["dw_gate"].dtype == grad and got["dx"].dtype == dtype
        want = _backward(x, wg, wu, dy, act, P, grad)
        for name, (value, error) in zip(("dx", "dw_gate", "dw_up"), want):
            within(got[name], value, error, (name, grad))
        again = _lm().gated_ffn_grad(x, wg, wu, dy, act=act, P=P, dtype=grad)
        assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("dtype,P,n,D,F", [
    (BF16, 1, 1, 4096, 5000), (BF16, 1, 16, 1024, 3000), (BF16, 1, 2048, 512, 2050),
    (BF16, 3, 700, 320, 1500), (F32, 1, 1500, 250, 1100), (F32, 7, 31, 1024, 513),
    (BF16, 1, 5, 9000, 70), (BF16, 1, 3000, 64, 8200)])
def test_larger(dtype, P, n, D, F):
    """Large tiles, products split along k, and several rounds of tiles."""
    announce("ffn, larger", dtype, P, n, D, F)
    x, wg, wu, dy = _inputs(P * n, D, F, dtype, 1)
    within(_lm().gated_ffn(x, wg, wu), *_forward(x, wg, wu, "silu"), "y")
    got = _lm().gated_ffn_grad(x, wg, wu, dy, P=P)
    want = _backward(x, wg, wu, dy, "silu", P, dtype)
    for name, (value, error) in zip(("dx", "dw_gate", "dw_up"), want):
        within(got[name], value, error, name)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,D,F", [
    (1, 4096, 6700), (16, 4096, 6400), (32, 4096, 300), (33, 4096, 300), (64, 4097, 260),
    (20, 2001, 3000), (40, 1000, 5100), (64, 136, 100)])
def test_few_rows(dtype, n, D, F):
    """Up to 64 rows on either side of where tiles take over, with the same bits
    at any alignment, in and out."""
    lm = _lm()
    announce("ffn, few rows", dtype, n, D, F)
    x, wg, wu, _ = _inputs(n, D, F, dtype, 21)
    for act in ("silu", "gelu"):
        y = lm.gated_ffn(x, wg, wu, act=act)
        within(y, *_forward(x, wg, wu, act), "y")

    def wide(t, gap, at):
        buf = torch.full((t.shape[0], t.shape[1] + gap), 7.0, dtype=dtype, device="cuda")
        buf[:, at:at + t.shape[1]] = t
        return buf, buf[:, at:at + t.shape[1]]
    sx, sg, su = (wide(t, 5, 3)[1] for t in (x, wg, wu))
    obuf, out = wide(torch.zeros_like(y), 3, 1)
    for args in ((sx, wg, wu), (x, sg, su), (sx, wg, su)):
        lm.gated_ffn(*args, act=act, out=out)
        assert torch.equal(out, y)
        out.fill_(7.0)
        assert (obuf == 7.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_alignments(dtype):
    """Rows with gaps, arrays at any element, outputs in wide buffers whose gaps
    stay, more leading dimensions; the same bits as dense operands give."""
    lm = _lm()
    P, n, D, F = 2, 37, 128, 70
    announce("ffn, strides", dtype)
    x, wg, wu, dy = _inputs(P * n, D, F, dtype, 2)
    y, want = lm.gated_ffn(x, wg, wu), lm.gated_ffn_grad(x, wg, wu, dy, P=P)

    def wide(t, gap, at):
        buf = torch.full((t.shape[0], t.shape[1] + gap), 7.0, dtype=dtype, device="cuda")
        buf[:, at:at + t.shape[1]] = t
        return buf, buf[:, at:at + t.shape[1]]
    for gap, at in ((3, 1), (8, 8), (64, 3)):
        sx, sg, su, sy = (wide(t, gap, at)[1] for t in (x, wg, wu, dy))
        obuf, out = wide(torch.zeros_like(y), gap, at)
        assert lm.gated_ffn(sx, sg, su, out=out) is out
        assert torch.equal(out, y)
        out.fill_(7.0)
        assert (obuf == 7.0).all()
        xbuf, dx = wide(torch.zeros_like(x), gap, at)
        # workers' gradients inside of wider contributions
        flat = torch.full((P, 2 * F * D + 11), 7.0, dtype=dtype, device="cuda")
        dwg = flat[:, 5:5 + F * D].unflatten(1, (F, D))
        dwu = flat[:, 6 + F * D:6 + 2 * F * D].unflatten(1, (F, D))
        got = lm.gated_ffn_grad(sx, sg, su, sy, P=P, dx=dx, dw_gate=dwg, dw_up=dwu)
        assert all(torch.equal(got[k], want[k]) for k in want)
        for t in (dx, dwg, dwu):
            t.fill_(7.0)
        assert (xbuf == 7.0).all() and (flat == 7.0).all()
        # one matrix with gaps beside one without
        assert torch.equal(lm.gated_ffn(x, wg, su), y)
    shaped = lm.gated_ffn(x.view(P, n, D), wg, wu)
    assert torch.equal(shaped, y.view(P, n, F))


@pytest.mark.parametrize("dtype,grad", [(BF16, BF16), (BF16, F32), (F32, F32)])
def test_accumulate(dtype, grad):
    lm = _lm()
    P, n, D, F = 3, 50, 96, 33
    announce("ffn, accumulate", dtype, grad)
    x, wg, wu, dy = _inputs(P * n, D, F, dtype, 3)
    g = torch.Generator().manual_seed(9)
    old = [torch.randn((P, F, D), generator=g).to(grad).cuda() for _ in range(2)]
    new = [t.clone() for t in old]
    lm.gated_ffn_grad(x, wg, wu, dy, P=P, dw_gate=new[0], dw_up=new[1], accumulate=True)
    want = _backward(x, wg, wu, dy, "silu", P, grad)[1:]
    for got, was, (value, error), name in zip(new, old, want, ("dw_gate", "dw_up")):
        # one more addition in fp32
        value = value + was.double()
        within(got, value, error + 2 * U * (value.abs() + error), name)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_rows(dtype):
    """Without rows the weights' gradients are zeros, or stay with accumulate."""
    lm = _lm()
    announce("ffn, no rows", dtype)
    wg = torch.ones((5, 7), dtype=dtype, device="cuda")
    x, dy = torch.zeros((0, 7), dtype=dtype, device="cuda"), torch.zeros((0, 5), dtype=dtype,
                                                                       device="cuda")
    assert lm.gated_ffn(x, wg, wg).shape == (0, 5)
    for P in (1, 3):
        got = lm.gated_ffn_grad(x, wg, wg, dy, P=P)
        assert got["dx"].shape == (0, 7)
        assert all(got[k].shape == (P, 5, 7) and (got[k] == 0).all() for k in ("dw_gate", "dw_up"))
        one = [torch.ones((P, 5, 7), dtype=dtype, device="cuda") for _ in range(2)]
        lm.gated_ffn_grad(x, wg, wg, dy, P=P, dw_gate=one[0], dw_up=one[1], accumulate=True)
        assert all((t == 1).all() for t in one)


def test_many_workers():
    """Workers of one row each, padded to 64: dg and du in their other order, in
    three pieces, take more workgroups than one launch has."""
    lm = _lm()
    P, F = 44500, 4032
    announce("ffn, many workers", P, F)
    assert 6 * P * (F // 64) * 256 >= 2 ** 32
    if torch.cuda.mem_get_info()[0] < (170 << 30):
        pytest.skip("not enough memory")
    x, wg, wu, dy = _inputs(P, 1, F, BF16, 22)
    got = lm.gated_ffn_grad(x, wg, wu, dy, P=P, dtype=F32)
    # _backward's formulas, for products of one term
    a, ea, da, eda, u, eu = _projections(x, wg, wu, "silu")
    x, dy = x.double(), dy.double()
    dg, du = dy * u * da, dy * a
    edg = dy.abs() * (eu * (da.abs() + eda) + u.abs() * eda) + 4 * U * dg.abs()
    edu = dy.abs() * ea + 4 * U * du.abs()
    for name, d, e in (("dw_gate", dg, edg), ("dw_up", du, edu)):
        error = (product_error(1, F32) * (d.abs() + e) + e) * x.abs()
        bad = (got[name][:, :, 0].double() - d * x).abs() > error + ULP[F32] * (d * x).abs() + 2.0 ** -120
        assert not bad.any(), (name, int(bad.sum()))
    del got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradient_against_differences(act):
    """Central differences of the forward call along random directions, in fp32:
    y is off by some D u relative, steps of 2^-6 leave (2^-6)^2 of the third
    derivative; 1e-3 of the sums' scale is above both."""
    lm = _lm()
    announce("ffn, differences", act)
    x, wg, wu, dy = _inputs(40, 60, 50, F32, 4)
    g = lm.gated_ffn_grad(x, wg, wu, dy, act=act)
    gen = torch.Generator().manual_seed(3)
    step = 2.0 ** -6
    for k, grad in enumerate((g["dx"], g["dw_gate"][0], g["dw_up"][0])):
        v = torch.randn(grad.shape, generator=gen).cuda() * (1.0 if k == 0 else 0.1)

        def at(h):
            args = [x, wg, wu]
            args[k] = args[k] + h * v
            return (lm.gated_ffn(*args, act=act).double() * dy.double()).sum()
        slope = float(at(step) - at(-step)) / (2 * step)
        want = float((grad.double() * v.double()).sum())
        assert abs(slope - want) <= 1e-3 * float((grad.double() * v.double()).norm()) * 8 + 1e-3


def test_large_and_lost_values():
    """Saturated activations, zero and infinite inputs of one row only: the other
    rows' results are unchanged."""
    lm = _lm()
    announce("ffn, large values")
    for dtype in (BF16, F32):
        for act in ("silu", "gelu"):
            x, wg, wu, _ = _inputs(70, 64, 40, dtype, 5)
            y = lm.gated_ffn(x * 100, wg, wu, act=act)
            within(y, *_forward(x * 100, wg, wu, act), "saturated")
            assert (lm.gated_ffn(torch.zeros_like(x), wg, wu, act=act) == 0).all()
            want = lm.gated_ffn(x, wg, wu, act=act)
            for bad in (math.inf, math.nan):
                z = x.clone()
                z[11, 3] = bad
                got = lm.gated_ffn(z, wg, wu, act=act)
                assert not torch.isfinite(got[11]).any()
                keep = torch.arange(70, device="cuda") != 11
                assert torch.equal(got[keep], want[keep])


def test_fp32_extremes():
    """fp32 operands near the ends of the range: three pieces hold the largest
    values, and small ones down to 2^-117."""
    lm = _lm()
    announce("ffn, fp32 extremes")
    one = torch.zeros((1, 64), device="cuda")
    one[0, 0] = 1.0
    big = torch.zeros((3, 64), device="cuda")
    big[:, 0] = torch.tensor([3.4028234e38, 1.0 + 2.0 ** -23, 2.0 ** -100 * (1 + 2.0 ** -23)])
    unit = torch.zeros((3, 64), device="cuda")
    unit[:, 0] = 1.0
    # act(large g) = g, so that y = u at g = 64
    y = lm.gated_ffn(one, unit * 64.0, big * (1.0 / 64.0))
    assert torch.equal(y[0].cpu(), (big[:, 0] / 64.0 * 64.0).cpu())


def test_on_another_stream_and_in_a_graph():
    lm = _lm()
    for P, n, D, F in ((2, 60, 96, 70), (1, 700, 512, 1300)):
        announce("ffn, stream and graph", P, n, D, F)
        x, wg, wu, dy = _inputs(P * n, D, F, BF16, 6)
        want_y, want = lm.gated_ffn(x, wg, wu), lm.gated_ffn_grad(x, wg, wu, dy, P=P, dtype=F32)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            y, got = lm.gated_ffn(x, wg, wu), lm.gated_ffn_grad(x, wg, wu, dy, P=P, dtype=F32)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(y, want_y) and all(torch.equal(got[k], want[k]) for k in got)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = lm.gated_ffn(x, wg, wu)
            got = lm.gated_ffn_grad(x, wg, wu, dy, P=P, dtype=F32)
        for k in range(3):
            x.copy_(_inputs(P * n, D, F, BF16, 7 + k)[0])
            graph.replay()
            torch.cuda.synchronize()
            want_y = lm.gated_ffn(x, wg, wu)
            want = lm.gated_ffn_grad(x, wg, wu, dy, P=P, dtype=F32)
            assert torch.equal(y, want_y) and all(torch.equal(got[i], want[i]) for i in got)


def test_single_rows_and_far_rows():
    """A vector, rows around the number that is taken without packing, and rows
    further apart than 32 bits reach."""
    lm = _lm()
    announce("ffn, single and far rows")
    for dtype in (BF16, F32):
        for N in (15, 16, 17, 32, 33, 48, 64, 65):
            x, wg, wu, _ = _inputs(N, 200, 90, dtype, 10)
            within(lm.gated_ffn(x, wg, wu), *_forward(x, wg, wu, "silu"), N)
        assert torch.equal(lm.gated_ffn(x[3], wg, wu), lm.gated_ffn(x[3:4], wg, wu)[0])
        got = lm.gated_ffn_grad(x[3], wg, wu, lm.gated_ffn(x[3], wg, wu))
        assert got["dx"].shape == (200,) and got["dw_gate"].shape == (1, 90, 200)
    pitch = (1 << 27) + 8
    for N in (40, 70):
        x, wg, wu, dy = _inputs(N, 64, 40, BF16, 11)
        y, want = lm.gated_ffn(x, wg, wu), lm.gated_ffn_grad(x, wg, wu, dy)
        far = torch.empty(N * pitch, dtype=BF16, device="cuda").view(N, pitch)
        wide = [far[:, 64 * i:64 * (i + 1)] for i in range(6)]
        wide[0].copy_(x)
        wide[1][:40].copy_(wg)
        wide[2][:40].copy_(wu)
        wide[3][:, :40].copy_(dy)
        args = wide[0], wide[1][:40], wide[2][:40]
        assert torch.equal(lm.gated_ffn(*args, out=wide[4][:, :40]), y)
        got = lm.gated_ffn_grad(*args, wide[3][:, :40], dx=wide[5])
        assert all(torch.equal(got[k], want[k]) for k in got)


def test_one_gradient():
    """dx alone, and the weights' alone, are what both together give."""
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("ffn, one gradient")
    P, n, D, F = 2, 70, 100, 90
    for dtype, kind in ((BF16, E.ECC_BF16), (F32, E.ECC_F32)):
        x, wg, wu, dy = _inputs(P * n, D, F, dtype, 12)
        want = lm.gated_ffn_grad(x, wg, wu, dy, P=P)
        a = E.ecc_ffn_t(n, D, F, P, kind, kind, E.ECC_ACT_SILU, x.data_ptr(), D, wg.data_ptr(), D,
                        wu.data_ptr(), D)
        work = torch.empty(E.ecc_ffn_work_size(a, 1), dtype=torch.uint8, device="cuda")
        stream = torch.cuda.current_stream().cuda_stream
        new = {k: torch.full_like(v, math.nan) for k, v in want.items()}
        E.ecc_ffn_grad(a, dy, F, new["dx"], D, None, None, 0, 0, work, stream)
        assert torch.equal(new["dx"], want["dx"])
        E.ecc_ffn_grad(a, dy, F, None, 0, new["dw_gate"], new["dw_up"], F * D, 0, work, stream)
        assert all(torch.equal(new[k], want[k]) for k in want)


def test_work_buffers():
    """A work buffer full of NaN changes nothing, and neither does its place;
    buffers that do not hold are refused."""
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("ffn, work buffers")
    for dtype in (BF16, F32):
        x, wg, wu, dy = _inputs(90, 100, 75, dtype, 8)
        y, want = lm.gated_ffn(x, wg, wu), lm.gated_ffn_grad(x, wg, wu, dy)
        work = torch.full((1 << 22,), math.nan, device="cuda")
        assert torch.equal(lm.gated_ffn(x, wg, wu, work=work[4:]), y)
        work.fill_(math.nan)
        got = lm.gated_ffn_grad(x, wg, wu, dy, work=work[8:])
        assert all(torch.equal(got[k], want[k]) for k in got)
        for bad in (work[:4], work.cpu(), work[::2]):
            with pytest.raises(ValueError):
                lm.gated_ffn_grad(x, wg, wu, dy, work=bad)
        with pytest.raises(E.EccError):
            lm.gated_ffn_grad(x, wg, wu, dy, work=work[1:])


def test_refusals():
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("ffn refusals")
    x, wg, wu, dy = _inputs(12, 16, 8, F32, 9)
    for args in ((x, wg[:, :15], wu), (x, wg, wu[:7]), (x[:, :8], wg, wu), (x.t(), wg, wu),
                 (x, wg.t(), wu.t())):
        with pytest.raises(ValueError):
            lm.gated_ffn(*args)
    for args in ((x.half(), wg, wu), (x.double(), wg.double(), wu.double()),
                 (x, wg.bfloat16(), wu.bfloat16()), (x, wg, wu.bfloat16())):
        with pytest.raises(TypeError):
            lm.gated_ffn(*args)
    with pytest.raises(ValueError):
        lm.gated_ffn(x, wg, wu, act="relu")
    with pytest.raises(ValueError):
        lm.gated_ffn(x, wg, wu, out=torch.empty((12, 9), device="cuda"))
    with pytest.raises(ValueError):
        lm.gated_ffn(x, wg, wu.cpu())
    with pytest.raises(ValueError):
        lm.gated_ffn(x.cpu(), wg.cpu(), wu.cpu())
    with pytest.raises(TypeError):
        lm.gated_ffn_grad(x, wg, wu, dy, dtype=F64)
    with pytest.raises(TypeError):
        lm.gated_ffn_grad(x, wg, wu, dy, dtype=BF16)
    d = torch.empty((2, 8, 16), device="cuda")
    for kw in (dict(P=5), dict(accumulate=True), dict(dw_gate=d[:1]), dict(P=2, dw_gate=d, dw_up=d[:1]),
               dict(dw_gate=d[:1], dw_up=d[:1, :, :8]), dict(dx=x[:11])):
        with pytest.raises(ValueError):
            lm.gated_ffn_grad(x, wg, wu, dy, **kw)
    with pytest.raises(ValueError):
        lm.gated_ffn_grad(x, wg, wu, dy[:11])

    def status(call):
        with pytest.raises(E.EccError) as e:
            call()
        return e.value.status
    # outputs over inputs and over each other
    assert status(lambda: lm.gated_ffn_grad(x, wg, wu, dy, dx=x)) == E.ECC_ERR_ARG
    assert status(lambda: lm.gated_ffn_grad(x, wg, wu, dy, dw_gate=d[:1], dw_up=d[:1])) == \
        E.ECC_ERR_ARG
    assert status(lambda: lm.gated_ffn_grad(x, wg, wu, dy, P=2, dw_gate=d, dw_up=d)) == \
        E.ECC_ERR_ARG
    sq = torch.randn((8, 8), device="cuda")
    assert status(lambda: lm.gated_ffn(sq, sq, sq, out=sq)) == E.ECC_ERR_ARG
