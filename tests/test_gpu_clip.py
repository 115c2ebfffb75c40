"""Global norms and clipping of gradients through the library's calls, against
the definition in 64 bits.

Tolerances (u = 2^-53).  Squares and their sums are formed in fp64: a sum of n
terms of one sign is within n u of itself, its root within half of that and u.
A scaled element is the product with max_norm / norm, both within the norm's
error and 2 u, rounded once to its type."""
import math

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


def _grads(shapes, types, P=None, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    lead = () if P is None else (P,)
    return [(torch.randn(lead + s, generator=g, dtype=F64) * scale).to(t).cuda()
            for s, t in zip(shapes, types)]


def _norms(grads, P):
    return torch.stack([g.double().cpu().reshape(P or 1, -1).square().sum(1)
                        for g in grads]).sum(0).sqrt()


def _near(got, want, n):
    assert ((got.cpu() - want).abs() <= (n + 8) * 2.0 ** -53 * want).all()


def _check(grads, max_norm, P=None, out_types=None, **kw):
    """In place where out_types is None, else into new tensors."""
    lm = _lm()
    n = sum(g.numel() for g in grads) // (P or 1)
    want = _norms(grads, P)
    by = torch.where(want > max_norm, max_norm / want, torch.ones((), dtype=F64))
    before = [g.clone() for g in grads]
    _near(lm.grad_norm(grads, P=P), want, n)
    out = None if out_types is None else [torch.full(g.shape, math.nan, dtype=t, device="cuda")
                                          for g, t in zip(grads, out_types)]
    norms = lm.clip_grads(grads, max_norm, P=P, out=out, **kw)
    _near(norms, want, n)
    for g, b, o in zip(grads, before, out or grads):
        b = b.double().cpu().reshape(P or 1, -1)
        exact = b * by[:, None]
        tol = (n + 12) * 2.0 ** -53 * exact.abs()
        tol = tol + ULP[o.dtype] * (exact.abs() + tol) + 1e-320
        got = o.double().cpu().reshape(P or 1, -1)
        if o.dtype != F64:       # (fp32's and bf16's smallest step)
            tol = tol + 2.0 ** -134
        assert ((got - exact).abs() <= tol).all()
        # workers within the limit keep their gradients, where the type holds
        # them (a narrower one has them rounded once, which torch's conversion
        # of fp64 to bf16, by way of fp32, does not give)
        same = (by == 1.0)
        if ULP[o.dtype] <= ULP[g.dtype]:
            assert torch.equal(got[same], b[same])
    if out is not None:
        assert all(torch.equal(g, b) for g, b in zip(grads, before))
    return norms


SHAPES = [(1,), (3, 5), (64,), (7, 129), (0, 4), (1000,), (33, 257), (4097,)]


@pytest.mark.parametrize("types", [(F32,), (BF16,), (F64,), (F32, BF16, F64)])
@pytest.mark.parametrize("P", [None, 1, 3, 16])
def test_small(types, P):
    announce("clip", types, P)
    kinds = [types[i % len(types)] for i in range(len(SHAPES))]
    for limit in (0.5, 1e9, 0.0):
        grads = _grads(SHAPES, kinds, P, 1)
        _check(grads, limit, P)
        for out in (F32, BF16, F64):
            _check(_grads(SHAPES, kinds, P, 2), limit, P, [out] * len(SHAPES))
    # each worker by its own norm
    if P and P > 1:
        grads = _grads(SHAPES, kinds, P, 3)
        size = torch.logspace(-2, 2, P, dtype=F64).cuda()
        grads = [(g.double() * size.view((P,) + (1,) * (g.dim() - 1))).to(g.dtype) for g in grads]
        limit = float(_norms(grads, P).median())
        _check(grads, limit, P)


@pytest.mark.parametrize("shapes,types,P", [
    ([(5000, 1003), (77,), (3, 3)], (F32, F32, F32), None),
    ([(300, 1003), (77,), (2000, 700)], (BF16, F32, F64), 5),
    ([(1 << 23,)], (BF16,), None), ([(3,)] * 300, (F32,) * 300, 2),
    ([(i % 7,) for i in range(500)], (BF16, F64) * 250, None)])
def test_larger(shapes, types, P):
    """Chunks that end inside a tensor, sums added in a launch of their own,
    more tensors than one launch describes."""
    announce("clip, larger", len(shapes), shapes[0], P)
    _check(_grads(shapes, types, P, 4), 1.5, P)
    _check(_grads(shapes, types, P, 4), 1.5, P, [F64] * len(shapes))
    a = _lm().grad_norm(_grads(shapes, types, P, 4), P=P)
    assert torch.equal(a, _lm().grad_norm(_grads(shapes, types, P, 4), P=P))


def test_range():
    """Squares beyond fp32's range on both sides."""
    announce("clip, range")
    for value in (1e30, 3e38, 1e-30, 1e-42):
        for dtype in (F32, BF16):
            g = [torch.full((300, 7), value, dtype=dtype, device="cuda")]
            exact = float(g[0][0, 0].double()) * math.sqrt(2100)
            norms = _lm().grad_norm(g)
            assert abs(float(norms) - exact) <= 1e-12 * exact
    g = [torch.full((1000,), 1e38, device="cuda")]
    _check(g, 1.0)
    g = [torch.full((1000,), 1e-300, dtype=F64, device="cuda")]
    assert float(_lm().clip_grads(g, 1.0)) == 0.0 and (g[0] == 1e-300).all()


def test_norms_that_are_not_finite():
    """Infinities and NaN of one worker: kept as they are, or zeros; the others
    are clipped as ever."""
    lm = _lm()
    announce("clip, not finite")
    for bad in (math.inf, -math.inf, math.nan):
        for dtype in (F32, BF16, F64):
            grads = _grads([(40, 9), (1001,)], (dtype, dtype), 3, 5)
            want = [g.clone() for g in grads]
            lm.clip_grads(want, 0.25, P=3)
            for t in (grads, want):
                t[1][1, 500] = bad
            for nonfinite in ("keep", "zero"):
                got = [g.clone() for g in grads]
                norms = lm.clip_grads(got, 0.25, P=3, nonfinite=nonfinite)
                assert torch.isfinite(norms).tolist() == [True, False, True]
                for k in (0, 1):
                    assert torch.equal(got[k][0], want[k][0]) and torch.equal(got[k][2], want[k][2])
                    if nonfinite == "zero":
                        assert (got[k][1] == 0).all()
                    else:
                        assert torch.equal(got[k][1].nan_to_num(3.0), grads[k][1].nan_to_num(3.0))
                out = [torch.full(g.shape, 5.0, dtype=F64, device="cuda") for g in grads]
                lm.clip_grads(grads, 0.25, P=3, out=out, nonfinite=nonfinite)
                for o, g in zip(out, got):
                    assert torch.equal(o[1].nan_to_num(3.0), g[1].double().nan_to_num(3.0))


def test_into_contributions():
    """Parameters' places in the workers' contributions, fp64, at odd elements;
    what lies between them stays; places and separate tensors mixed."""
    lm = _lm()
    announce("clip, contributions")
    P, shapes = 4, [(31, 7), (1,), (513,), (20, 20)]
    grads = _grads(shapes, [F32] * 4, P, 6)
    sizes = [math.prod(s) for s in shapes]
    flat = torch.full((P, sum(sizes) + 9), 7.0, dtype=F64, device="cuda")
    out, at = [], 3
    for s, n in zip(shapes, sizes):
        out.append(flat[:, at:at + n].unflatten(1, s))
        at += n + 1
    want = _norms(grads, P)
    lm.clip_grads(grads, 1.0, P=P, out=out)
    for g, o in zip(grads, out):
        exact = g.double() * (1.0 / want).cuda().view((P,) + (1,) * (g.dim() - 1))
        assert ((o - exact).abs() <= 1e-12 * exact.abs()).all()
        o.fill_(7.0)
    assert (flat == 7.0).all()
    # in place within contributions, and None for some
    out[0].copy_(grads[0])
    keep = grads[1].clone()
    lm.clip_grads([out[0], grads[1], grads[2]], 1.0, P=P, out=[None, None, out[2]])
    part = _norms([grads[0], keep, grads[2]], P)
    by = (1.0 / part).clamp(max=1.0).cuda()
    assert ((out[0] - grads[0].double() * by[:, None, None]).abs() <= 1e-12).all()
    assert ((grads[1].double() - keep.double() * by[:, None]).abs() <= 1e-6 * keep.abs()).all()


@pytest.mark.parametrize("wide_out", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_out_of_contributions(dtype, wide_out):
    """Gradients within one buffer of all workers', as the feed-forward block and
    cross entropy write them, clipped into dense tensors and into places of
    another pitch; what lies around the outputs stays."""
    lm = _lm()
    announce("clip, out of contributions", dtype, wide_out)
    P, shapes = 3, [(31, 7), (1,), (5000,), (2, 10)]
    sizes = [math.prod(s) for s in shapes]
    wide = torch.zeros((P, 2 * sum(sizes)), dtype=dtype, device="cuda")
    grads, at = [], 5
    for dense, s, n in zip(_grads(shapes, [dtype] * 4, P, 11), shapes, sizes):
        grads.append(wide[:, at:at + n].unflatten(1, s))
        grads[-1].copy_(dense)
        at += n + 3
    want = _norms(grads, P)
    for out_type in (F32, F64):
        # (room for a worker's elements at any of the gradients' distances)
        room = P * wide.shape[1] + 64
        bufs, out = [], []
        for s, n in zip(shapes, sizes):
            bufs.append(torch.full((room,), 7.0, dtype=out_type, device="cuda"))
            pitch = n + 11 if wide_out else n
            out.append(bufs[-1][16:16 + P * pitch].view(P, pitch)[:, :n].unflatten(1, s))
            assert out[-1].is_contiguous() != wide_out
        _near(lm.clip_grads(grads, 1.0, P=P, out=out), want, sum(sizes))
        for g, o, buf in zip(grads, out, bufs):
            exact = g.double() * (1.0 / want).cuda().view((P,) + (1,) * (g.dim() - 1))
            tol = ULP[out_type] * exact.abs() + 1e-12 * exact.abs()
            assert ((o.double() - exact).abs() <= tol).all()
            o.fill_(7.0)
            assert (buf == 7.0).all()


def test_alignments():
    """Tensors at every element of 16 bytes, of every length around the vectors'."""
    lm = _lm()
    announce("clip, alignments")
    for dtype in (F32, BF16, F64):
        buf = torch.randn(20000, generator=torch.Generator().manual_seed(7), dtype=F64).to(
            dtype).cuda()
        for at in range(0, 9):
            for n in (1, 7, 8, 9, 4095, 4096, 4097, 8193):
                g = [buf[at:at + n]]
                want = float(g[0].double().norm())
                o = torch.full((n + 2,), 7.0, dtype=F32, device="cuda")
                norms = lm.clip_grads(g, want / 2, out=[o[1:-1]])
                assert abs(float(norms) - want) <= (n + 8) * 2.0 ** -52 * want
                assert (o[1:-1].double() - g[0].double() / 2).abs().max() <= 2.0 ** -24 * 8
                assert o[0] == 7 and o[-1] == 7


def test_on_another_stream_and_in_a_graph():
    lm = _lm()
    for count in (5, 150):
        announce("clip, stream and graph", count)
        grads = _grads([(300, 17)] * count, [F32] * count, 2, 8)
        out = [torch.empty_like(g, dtype=F64) for g in grads]
        want_n = lm.clip_grads(grads, 1.0, P=2, out=out)
        want = [o.clone() for o in out]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got_n = lm.clip_grads(grads, 1.0, P=2, out=out)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got_n, want_n) and all(torch.equal(a, b) for a, b in zip(out, want))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got_n = lm.clip_grads(grads, 1.0, P=2, out=out)
            alone = lm.grad_norm(grads, P=2)
        for k in range(3):
            for g in grads:
                g.mul_(1.5 + k)
            graph.replay()
            torch.cuda.synchronize()
            got = [o.clone() for o in out]
            want_n = lm.clip_grads(grads, 1.0, P=2, out=out)
            assert torch.equal(got_n, want_n) and torch.equal(alone, want_n)
            assert all(torch.equal(a, b) for a, b in zip(out, got))


def test_work_buffers():
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("clip, work buffers")
    for count in (3, 70):
        grads = _grads([(500,)] * count, [F32] * count, None, 9)
        want = lm.grad_norm(grads)
        work = torch.full((1 << 14,), math.nan, device="cuda")
        assert torch.equal(lm.grad_norm(grads, work=work[4:]), want)
        with pytest.raises(E.EccError):
            lm.grad_norm(grads, work=work[1:])
        for bad in (work[:1], work.cpu(), work[::2]):
            with pytest.raises(ValueError):
                lm.clip_grads(grads, 1.0, work=bad)


def test_refusals():
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("clip refusals")
    g = _grads([(4, 6), (5,)], [F32, F32], None, 10)
    p = _grads([(4, 6), (5,)], [F32, F32], 3, 10)
    for args, kw in (((p,), dict(P=2)), (([],), {}), ((g,), dict(P=0)), (([g[0].t()],), {}),
                     (([g[0].cpu()],), {}), (([g[0], g[1].cpu()],), {}),
                     (([p[0].transpose(0, 1)],), dict(P=4)), ((g,), dict(norms=p[0][0, 0, :1]))):
        with pytest.raises(ValueError):
            lm.grad_norm(*args, **kw)
    with pytest.raises(TypeError):
        lm.grad_norm([g[0].half()])
    for out in ([g[0]], [g[0], p[1]], [g[1], g[0]], [g[0].cpu(), None]):
        with pytest.raises(ValueError):
            lm.clip_grads(g, 1.0, out=out)
    with pytest.raises(ValueError):
        lm.clip_grads(g, 1.0, nonfinite="drop")

    def status(*args, **kw):
        with pytest.raises(E.EccError) as e:
            lm.clip_grads(*args, **kw)
        return e.value.status
    for limit in (-1.0, math.nan):
        assert status(g, limit) == E.ECC_ERR_ARG
    buf = torch.zeros(64, device="cuda")
    # an output over another gradient, two outputs in one place, a gradient twice
    assert status([buf[:8], buf[8:16]], 1.0, out=[buf[8:16], None]) == E.ECC_ERR_ARG
    assert status([buf[:8], buf[8:16]], 1.0, out=[buf[32:40], buf[39:47]]) == E.ECC_ERR_ARG
    assert status([buf[:8], buf[:8]], 1.0) == E.ECC_ERR_ARG
    assert status([buf[:8]], 1.0, out=[buf[4:12]]) == E.ECC_ERR_ARG
    # in place as another type
    wide = buf.view(F64)
    assert status([buf[:32]], 1.0, out=[wide[:32]]) == E.ECC_ERR_ARG
    # workers of one tensor over each other, places that overlap within contributions
    flat = torch.zeros((3, 64), device="cuda")
    three = [torch.zeros((3, 8), device="cuda") for _ in range(2)]
    assert status(three, 1.0, P=3, out=[flat[:, :8], flat[:, 7:15]]) == E.ECC_ERR_ARG
    assert status([buf.as_strided((3, 8), (4, 1))], 1.0, P=3) == E.ECC_ERR_ARG
    assert status([flat[:, :8], flat[:, 8:16]], 1.0, P=3, out=[flat[:, 8:16], None]) == E.ECC_ERR_ARG
    lm.clip_grads(three, 1.0, P=3, out=[flat[:, :8], flat[:, 8:16]])
    lm.grad_norm([buf[:8], buf[:8]])
