"""Cross entropy from hidden states through the library's call, loss and
gradients, against the definition in 64 bits.

Tolerances (u = 2^-24; products as in product_bounds.py).  With a row's logits
off by up to e = max e_j + 2 u max |z_j| (the scale's product) and spread over X,
its exponentials are off by (2.2 X + 2) u more (X + 1.2 X of the difference and
the exponent; beyond X = 104 they are 0), and their sum by 2 e + (2 X + 64 + V /
64) u relative in all (the rest of X, the additions of 64 columns in 18 steps,
their joins in a wave of 64).  So the loss is within w (3 e + k u (1 + |lse -
z_y| + |z|)), k = 2 X + 64 + V / 64, and a softmax value within p (4 e + 2 k u).
dz is off by scale * w times that and 4 u of both its terms, and is stored with half a step of bf16
where a gradient is bf16, or as three pieces (none)."""
import math

import pytest

torch = pytest.importorskip("torch")

from gpu_common import announce                                        # noqa: E402
from product_bounds import BF16, F32, F64, U, ULP, product, within     # noqa: E402

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


def _inputs(N, D, V, dtype, seed=0, weight=True, size=1.5):
    g = torch.Generator().manual_seed(1000 * seed + N + 3 * D + 7 * V)
    h = torch.randn((N, D), generator=g, dtype=F64).to(dtype)
    table = (torch.randn((V, D), generator=g, dtype=F64) * size / math.sqrt(D)).to(dtype)
    y = torch.randint(-1, V + 1, (N,), generator=g).to(torch.int32)
    w = torch.rand((N,), generator=g) + 0.5
    w[torch.rand((N,), generator=g) < 0.2] = 0.0
    return h.cuda(), table.cuda(), y.cuda(), w.cuda() if weight else None


def _reference(h, table, y, w, scale, P, grad):
    """Loss, dh and dtable, each with the bound of its error."""
    t, (N, D), V = h.dtype, h.shape, table.shape[0]
    z, e = product(h.double(), table.double().t(), t)
    z, e = z * scale, e * abs(scale)
    known = (y >= 0) & (y < V)
    at = y.long().clamp(0, V - 1)[:, None]
    w = torch.ones(N, dtype=F64, device="cuda") if w is None else w.double()
    w = (w * known)[:, None]
    most = z.abs().amax(1, keepdim=True)
    e = e.amax(1, keepdim=True) + 2 * U * most
    X = z.amax(1, keepdim=True) - z.amin(1, keepdim=True)
    k = 2 * X + 64 + V / 64
    nll = torch.logsumexp(z, 1, keepdim=True) - z.gather(1, at)
    loss = w * nll
    el = w.abs() * (3 * e + k * U * (1 + nll.abs() + most))
    p = torch.softmax(z, 1)
    hot = torch.zeros_like(p).scatter_(1, at, 1.0)
    f = w * scale
    dz = f * (p - hot)
    ez = f.abs() * (p * (4 * e + 2 * k * U) + 4 * U * (p + hot))

    def stored(out):
        return ez + (ULP[BF16] * (dz.abs() + ez) if t == BF16 and out == BF16 else 0.0)
    dh = product(dz, table.double(), t, stored(t))
    n = N // P
    kind = F32 if grad == F32 else t    # (dz as three pieces: three products)
    parts = [product(dz[r].t(), h[r].double(), kind, stored(grad)[r].t())
             for r in (slice(q * n, (q + 1) * n) for q in range(P))]
    return ((loss[:, 0], el[:, 0]), dh, tuple(torch.stack(v) for v in zip(*parts)))


def _check(h, table, y, w=None, scale=1.0, P=1, dtype=None, **kw):
    got = _lm().cross_entropy(h, table, y, w, scale=scale, P=P, dtype=dtype, **kw)
    want = _reference(h, table, y, w, scale, P, dtype or h.dtype)
    assert got[0].dtype == F32 and got[1].dtype == h.dtype and got[2].dtype == (dtype or h.dtype)
    for g, (value, error), name in zip(got, want, ("loss", "dh", "dtable")):
        within(g, value, error, (name, dtype))
    again = _lm().cross_entropy(h, table, y, w, scale=scale, P=P, dtype=dtype)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    loss, dh, dtable = _lm().cross_entropy(h, table, y, w, scale=scale, grad=None)
    # (the loss alone may take other tiles, with the same sums)
    assert dh is None and dtable is None
    within(loss, *want[0], "loss alone")
    return got


SIZES = [(1, 1, 1, 1), (1, 1, 1, 2), (1, 3, 7, 5), (1, 61, 96, 1003), (2, 33, 65, 129),
         (3, 64, 128, 64), (5, 13, 250, 300), (4, 1, 40, 70), (1, 300, 130, 257), (1, 70, 63, 4000)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("P,n,D,V", SIZES)
def test_small(dtype, P, n, D, V):
    announce("cross entropy", dtype, P, n, D, V)
    h, table, y, w = _inputs(P * n, D, V, dtype)
    _check(h, table, y, w, P=P)
    _check(h, table, y, None, scale=0.3, P=P, dtype=F32)


@pytest.mark.parametrize("dtype,P,n,D,V,grad", [
    (BF16, 1, 1, 2048, 20000, BF16), (BF16, 1, 700, 520, 9000, F32), (BF16, 4, 700, 320, 3000, BF16),
    (F32, 1, 700, 250, 3001, F32), (F32, 7, 31, 1024, 513, F32), (BF16, 1, 20, 64, 100001, BF16),
    (BF16, 1, 5000, 64, 700, BF16), (BF16, 1, 2000, 700, 600, F32)])
def test_larger(dtype, P, n, D, V, grad):
    """Large tiles, products split along k, and several rounds of tiles."""
    announce("cross entropy, larger", dtype, P, n, D, V)
    _check(*_inputs(P * n, D, V, dtype, 1), P=P, dtype=grad)


def test_labels_and_weights():
    """Rows without a label or of weight 0 give zeros whatever they hold, all
    rows too; negative weights count."""
    lm = _lm()
    announce("cross entropy, labels and weights")
    for dtype in (BF16, F32):
        N, D, V = 150, 40, 333
        h, table, y, w = _inputs(N, D, V, dtype, 2)
        want = lm.cross_entropy(h, table, y, w)
        dead = (w == 0) | (y < 0) | (y >= V)
        assert 10 < int(dead.sum()) < N - 10
        z = h.clone()
        z[dead] = math.nan
        got = lm.cross_entropy(z, table, y, w)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert (got[0][dead] == 0).all() and (got[1][dead] == 0).all()
        none = torch.full_like(y, -100)
        for args in ((z, table, none, w), (z, table, y, torch.zeros_like(w))):
            got = lm.cross_entropy(*args)
            assert all((t == 0).all() for t in got)
            assert (lm.cross_entropy(*args, grad=None)[0] == 0).all()
        _check(h, table, y, w - 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_logits(dtype):
    """Logits up to some hundreds either way, and rows that are sure of their
    label."""
    announce("cross entropy, large logits", dtype)
    h, table, y, w = _inputs(60, 64, 500, dtype, 3, size=60.0)
    _check(h, table, y, w)
    _check(h, table, y, w, scale=-1.0)
    known = (y >= 0) & (y < 500)
    h = torch.where(known[:, None], table[y.long().clamp(0, 499)] * 0.1, h)
    loss = _check(h, table, y, w)[0]
    assert (loss[known & (w > 0)] >= 0).all()


@pytest.mark.parametrize("P,n,V", [(1, 70, 300), (1, 70, 2500), (1, 40, 300), (1, 40, 2500),
                                   (2, 9, 2500), (2, 100, 500)])
def test_small_probabilities(P, n, V):
    """fp32 probabilities down to e^-66, each to fp32's precision.  One row counts,
    whose logits are the table's column itself: its gradient in the table is
    softmax - [label], where the exponential is off by 4 u (2 ulp), the sum by 2
    u (the other terms are below 1e-8 in all), its inverse by 2 u, their product
    and the stored sum of three pieces by u each."""
    announce("cross entropy, small probabilities", P, n, V)
    table = -torch.linspace(24.0, 66.0, V, dtype=F64).to(F32).cuda()[:, None]
    table[0] = 0.0
    y = torch.full((P * n,), -1, dtype=torch.int32, device="cuda")
    y[-1] = 0
    h = torch.ones((P * n, 1), device="cuda")
    _, _, got = _lm().cross_entropy(h, table, y, P=P)
    # (on the CPU: the GPU's softmax in 64 bits is off by 3e-6 of its small values)
    want = torch.exp(table[:, 0].cpu().double())
    want /= want.sum()
    got = got[-1, :, 0].cpu().double()
    assert (got[1:] - want[1:]).abs().le(12 * U * want[1:]).all(), \
        float((got[1:] / want[1:] - 1).abs().max() / U)
    assert abs(float(got[0] - (want[0] - 1))) <= 8 * U


def test_rows_of_infinities():
    """A row whose hidden state is not finite spoils its own loss and gradient
    only, and the table's."""
    lm = _lm()
    announce("cross entropy, infinities")
    for dtype in (BF16, F32):
        h, table, y, w = _inputs(90, 64, 200, dtype, 4, weight=False)
        y.clamp_(0, 199)
        want = lm.cross_entropy(h, table, y)
        z = h.clone()
        z[17, 5] = math.inf
        got = lm.cross_entropy(z, table, y)
        keep = torch.arange(90, device="cuda") != 17
        assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1][keep], want[1][keep])
        assert not torch.isfinite(got[0][17])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_alignments(dtype):
    """Rows with gaps, arrays at any element, outputs in wide buffers whose gaps
    stay, more leading dimensions; the same bits as dense operands give."""
    lm = _lm()
    P, n, D, V = 2, 45, 128, 150
    announce("cross entropy, strides", dtype)
    h, table, y, w = _inputs(P * n, D, V, dtype, 5)
    want = lm.cross_entropy(h, table, y, w, P=P)

    def wide(t, gap, at):
        buf = torch.full((t.shape[0], t.shape[1] + gap), 7.0, dtype=dtype, device="cuda")
        buf[:, at:at + t.shape[1]] = t
        return buf, buf[:, at:at + t.shape[1]]
    for gap, at in ((3, 1), (8, 8), (64, 3)):
        sh, st = wide(h, gap, at)[1], wide(table, gap, at)[1]
        hbuf, dh = wide(torch.zeros_like(h), gap, at)
        flat = torch.full((P, V * (D + gap) + 11), 7.0, dtype=dtype, device="cuda")
        dt = flat[:, 5:5 + V * (D + gap)].unflatten(1, (V, D + gap))[..., :D]
        lbuf = torch.full((P * n + 2,), 7.0, device="cuda")
        got = lm.cross_entropy(sh, st, y, w, P=P, dh=dh, dtable=dt, loss=lbuf[1:-1])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        for t in (dh, dt, lbuf[1:-1]):
            t.fill_(7.0)
        assert all((t == 7.0).all() for t in (hbuf, flat, lbuf))
    got = lm.cross_entropy(h.view(P, n, D), table, y.view(P, n), w.view(P, n), P=P)
    assert torch.equal(got[0], want[0].view(P, n)) and torch.equal(got[1], want[1].view(P, n, D))


@pytest.mark.parametrize("dtype,grad", [(BF16, BF16), (BF16, F32), (F32, F32)])
def test_accumulate(dtype, grad):
    lm = _lm()
    P, n, D, V = 3, 50, 96, 133
    announce("cross entropy, accumulate", dtype, grad)
    h, table, y, w = _inputs(P * n, D, V, dtype, 6)
    y[n:2 * n] = -1     # (a worker without a row)
    g = torch.Generator().manual_seed(9)
    old = torch.randn((P, V, D), generator=g).to(grad).cuda()
    new = old.clone()
    lm.cross_entropy(h, table, y, w, P=P, dtable=new, accumulate=True)
    value, error = _reference(h, table, y, w, 1.0, P, grad)[2]
    value = value + old.double()
    within(new, value, error + 2 * U * (value.abs() + error), "dtable")
    assert torch.equal(new[1], old[1])
    # written, a worker without a row has zeros
    lm.cross_entropy(h, table, y, w, P=P, dtable=new)
    assert (new[1] == 0).all()


@pytest.mark.parametrize("dtype,grad,P", [(BF16, BF16, 1), (BF16, F32, 1), (BF16, BF16, 3)])
def test_several_pieces_of_rows(dtype, grad, P):
    """More logits than are held at a time: three pieces of rows, workers that
    lie in two of them, one whose rows do not count, added to what is there."""
    lm = _lm()
    n, D, V = 12000 // P, 64, 128000
    announce("cross entropy, pieces of rows", dtype, grad, P)
    h, table, y, w = _inputs(P * n, D, V, dtype, 7)
    if P > 1:
        y[n:2 * n] = -1
    old = torch.randn((P, V, D), generator=torch.Generator().manual_seed(2)).to(grad).cuda()
    new = old.clone()
    loss, dh, _ = lm.cross_entropy(h, table, y, w, P=P, dtable=new, accumulate=True)
    written = lm.cross_entropy(h, table, y, w, P=P, dtype=grad)[2]
    step = 1000
    total = torch.zeros((P, V, D), dtype=F64, device="cuda")
    error = torch.zeros_like(total)
    for r in range(0, P * n, step):
        rows = slice(r, r + step)
        want = _reference(h[rows], table, y[rows], w[rows], 1.0, 1, grad)
        within(loss[rows], *want[0], "loss")
        within(dh[rows], *want[1], "dh")
        total[r // n] += want[2][0][0]
        error[r // n] += want[2][1][0]
    # (the sum over all rows is one chain, and pieces are added in fp32)
    size = error + 2 * U * 12 * (total.abs() + error)
    within(written, total, 13 * size, "dtable")
    value = total + old.double()
    within(new, value, 13 * size + 2 * U * (value.abs() + size), "dtable, added to")


@pytest.mark.parametrize("dtype,grad", [(BF16, BF16), (BF16, F32), (F32, F32)])
def test_largest_vocabulary(dtype, grad):
    """As many tokens as are taken, of which 256 rows are a piece."""
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    N, D, V = 300, 3, E.ECC_CROSS_ENTROPY_MAX_VOCAB
    announce("cross entropy, largest vocabulary", dtype, grad)
    if torch.cuda.mem_get_info()[0] < (64 << 30):
        pytest.skip("not enough memory")
    h, table, y, w = _inputs(N, D, V, dtype, 24)
    y[7] = V - 1
    loss, dh, dtable = lm.cross_entropy(h, table, y, w, dtype=grad)
    total = torch.zeros((1, V, D), dtype=F64, device="cuda")
    error = torch.zeros_like(total)
    step = 30
    for r in range(0, N, step):
        rows = slice(r, r + step)
        want = _reference(h[rows], table, y[rows], w[rows], 1.0, 1, grad)
        within(loss[rows], *want[0], "loss")
        within(dh[rows], *want[1], "dh")
        total += want[2][0]
        error += want[2][1]
    # (the sum over all rows is one chain, and pieces are added in fp32)
    size = error + 2 * U * 10 * (total.abs() + error)
    within(dtable, total, 11 * size, "dtable")


def test_no_rows():
    lm = _lm()
    announce("cross entropy, no rows")
    for dtype in (BF16, F32):
        table = torch.ones((5, 7), dtype=dtype, device="cuda")
        h = torch.zeros((0, 7), dtype=dtype, device="cuda")
        y = torch.zeros(0, dtype=torch.int32, device="cuda")
        for P in (1, 3):
            loss, dh, dt = lm.cross_entropy(h, table, y, P=P)
            assert loss.shape == (0,) and dh.shape == (0, 7) and (dt == 0).all()
            one = torch.ones((P, 5, 7), dtype=dtype, device="cuda")
            lm.cross_entropy(h, table, y, P=P, dtable=one, accumulate=True)
            assert (one == 1).all()


@pytest.mark.parametrize("dtype,grad", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("n,D,V", [
    (1, 2, 1), (2, 64, 63), (15, 63, 64), (16, 65, 65), (17, 200, 2048), (31, 130, 2049),
    (32, 257, 1000), (33, 31, 640), (48, 1001, 90), (63, 128, 4001), (64, 96, 2113),
    (40, 2112, 700), (40, 2050, 2100)])
def test_few_rows(dtype, grad, n, D, V):
    """Up to 64 rows of one worker, whose operands are taken as they lie: blocks
    of 16 rows, 64 columns and 64 elements, tiles joined in one launch and in
    two, at any alignment; long rows of small vocabularies by tiles of a split
    product, packed and as they lie, with the same bits."""
    announce("cross entropy, few rows", dtype, grad, n, D, V)
    h, table, y, w = _inputs(n, D, V, dtype, 11)
    y[0], w[0] = V - 1, 0.7      # (a row that counts)
    want = _check(h, table, y, w, scale=-0.6, dtype=grad)
    for alike in (None, torch.full_like(w, 0.25)):
        _check(h, table, y, alike, dtype=grad)
    # rows with gaps, at any element; NaN in rows that do not count
    dead = (w == 0) | (y < 0) | (y >= V)

    def wide(t, rows):
        buf = torch.full((t.shape[0], D + 3), 7.0, dtype=t.dtype, device="cuda")
        buf[:, 1:1 + D] = t
        if rows is not None:
            buf[rows] = math.nan
        return buf, buf[:, 1:1 + D]
    outs = [wide(torch.zeros_like(t), None) for t in (h, want[2][0])]
    got = _lm().cross_entropy(wide(h, dead)[1], wide(table, None)[1], y, w, scale=-0.6,
                              dh=outs[0][1], dtable=outs[1][1][None], accumulate=True)
    # (added to zeros)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for buf, view in outs:
        view.fill_(7.0)
        assert (buf == 7.0).all()


@pytest.mark.parametrize("dtype,grad", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("P,n,D,V", [
    (2, 32, 64, 100), (64, 1, 70, 130), (3, 21, 33, 2100), (9, 7, 129, 63), (2, 3, 640, 2500),
    (6, 10, 2112, 300)])
def test_few_rows_of_workers(dtype, grad, P, n, D, V):
    """Up to 64 rows of several workers: each one's table gradient from its rows
    alone, alike or different weights, one whose rows do not count, added to what
    is there, and NaN and infinities in another worker's rows."""
    lm = _lm()
    announce("cross entropy, few rows of workers", dtype, grad, P, n, D, V)
    h, table, y, w = _inputs(P * n, D, V, dtype, 23)
    y[:n] = -1
    y[n], w[n] = V - 1, 0.6
    want = _check(h, table, y, w, P=P, dtype=grad)
    assert (want[2][0] == 0).all()
    own = torch.arange(1, P + 1, device="cuda").repeat_interleave(n) / (2.0 * P)
    _check(h, table, y, own.float(), scale=-1.5, P=P, dtype=grad)
    gap = torch.full((P, V + 2, D + 3), 7.0, dtype=grad, device="cuda")
    dt = gap[:, 1:V + 1, 2:D + 2]
    dt.zero_()
    dt[0] = -0.0
    got = lm.cross_entropy(h, table, y, w, P=P, dtable=dt, accumulate=True)
    assert torch.equal(got[2], want[2]) and torch.signbit(dt[0]).all()
    dt.fill_(7.0)
    assert (gap == 7.0).all()
    bad = h.clone()
    bad[n, 0], bad[2 * n - 1, D - 1] = math.inf, math.nan
    got = lm.cross_entropy(bad, table, y, w, P=P, dtype=grad)
    keep = torch.arange(P, device="cuda") != 1
    assert torch.equal(got[2][keep], want[2][keep])
    assert torch.equal(got[1].view(P, n, D)[keep], want[1].view(P, n, D)[keep])


@pytest.mark.parametrize("dtype,grad,n,D,V", [
    (BF16, BF16, 50, 130, 700), (BF16, F32, 9, 520, 2500), (F32, F32, 33, 70, 400),
    (BF16, BF16, 60, 2048, 500), (F32, F32, 40, 2050, 300)])
def test_few_rows_calls(dtype, grad, n, D, V):
    """Either gradient alone, a work buffer full of NaN of which nothing behind
    its size is touched, and replayed graphs, down to no row that counts."""
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("cross entropy, few rows' calls", dtype, grad, n, D, V)
    h, table, y, w = _inputs(n, D, V, dtype, 17)
    want = lm.cross_entropy(h, table, y, w, dtype=grad)
    kinds = {BF16: E.ECC_BF16, F32: E.ECC_F32}
    a = E.ecc_cross_entropy_t(n, V, D, 1, kinds[dtype], kinds[grad], 0, h.data_ptr(), D,
                              table.data_ptr(), D, y.data_ptr(), w.data_ptr(), 1.0)
    stream = torch.cuda.current_stream().cuda_stream
    for which in (0, 1, 2, 3):
        size = E.ecc_cross_entropy_work_size(a, 1 if which else 0)
        work = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
        loss = torch.full_like(want[0], math.nan)
        dh = torch.full_like(want[1], math.nan) if which & 1 else None
        dt = torch.full_like(want[2], math.nan) if which & 2 else None
        E.ecc_cross_entropy(a, loss, dh, D, dt, D, V * D, 0, work, stream)
        if which:
            for got, all_of_it in ((loss, want[0]), (dh, want[1]), (dt, want[2])):
                assert got is None or torch.equal(got, all_of_it)
        else:
            # (tiles are joined by 64 lanes where there is the loss alone, by four
            # where there are gradients and up to 32 tiles)
            within(loss, *_reference(h, table, y, w, 1.0, 1, grad)[0], "loss alone")
        assert (work[size:] == 255).all()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lm.cross_entropy(h, table, y, w, dtype=grad)
    for k in range(4):
        h2, _, y2, w2 = _inputs(n, D, V, dtype, 18 + k)
        h.copy_(h2)
        y.copy_(y2 if k < 3 else torch.full_like(y2, -1))
        w.copy_(w2)
        graph.replay()
        torch.cuda.synchronize()
        want = lm.cross_entropy(h, table, y, w, dtype=grad)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        if k == 3:
            assert all((t == 0).all() for t in got)
            old = torch.full_like(want[2], -0.0)
            lm.cross_entropy(h, table, y, w, dtable=old, accumulate=True)
            assert torch.signbit(old).all()      # (left alone)


def test_gradient_against_differences():
    """Central differences of the loss along random directions, in fp32."""
    lm = _lm()
    announce("cross entropy, differences")
    h, table, y, w = _inputs(80, 60, 300, F32, 8)
    _, dh, dt = lm.cross_entropy(h, table, y, w, scale=0.7)
    gen = torch.Generator().manual_seed(3)
    step = 2.0 ** -5
    for k, grad in enumerate((dh, dt[0])):
        v = torch.randn(grad.shape, generator=gen).cuda() * (1.0 if k == 0 else 0.1)

        def at(s):
            args = [h, table]
            args[k] = args[k] + s * v
            return lm.cross_entropy(*args, y, w, scale=0.7, grad=None)[0].double().sum()
        slope = float(at(step) - at(-step)) / (2 * step)
        want = float((grad.double() * v.double()).sum())
        # (losses of some 6 add to 500, each off by 1e-6; the third derivative
        # along v is of the order of |v . dz|^3 per row)
        assert abs(slope - want) <= 2e-2 + 2e-3 * abs(want)


def test_on_another_stream_and_in_a_graph():
    lm = _lm()
    for P, n, D, V in ((2, 60, 96, 700), (1, 900, 512, 4000)):
        announce("cross entropy, stream and graph", P, n, D, V)
        h, table, y, w = _inputs(P * n, D, V, BF16, 9)
        want = lm.cross_entropy(h, table, y, w, P=P, dtype=F32)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = lm.cross_entropy(h, table, y, w, P=P, dtype=F32)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = lm.cross_entropy(h, table, y, w, P=P, dtype=F32)
        for k in range(4):
            # (other rows that count, down to none)
            h2, _, y2, w2 = _inputs(P * n, D, V, BF16, 10 + k)
            h.copy_(h2)
            y.copy_(y2 if k < 3 else torch.full_like(y2, -1))
            w.copy_(w2)
            graph.replay()
            torch.cuda.synchronize()
            want = lm.cross_entropy(h, table, y, w, P=P, dtype=F32)
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_one_gradient():
    """Either gradient alone is what both calls together give."""
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("cross entropy, one gradient")
    P, n, D, V = 2, 70, 100, 333
    for dtype, kind in ((BF16, E.ECC_BF16), (F32, E.ECC_F32)):
        h, table, y, w = _inputs(P * n, D, V, dtype, 13)
        want = lm.cross_entropy(h, table, y, w, P=P)
        a = E.ecc_cross_entropy_t(n, V, D, P, kind, kind, 0, h.data_ptr(), D, table.data_ptr(), D,
                                  y.data_ptr(), w.data_ptr(), 1.0)
        work = torch.empty(E.ecc_cross_entropy_work_size(a, 1), dtype=torch.uint8, device="cuda")
        stream = torch.cuda.current_stream().cuda_stream
        for which in (1, 2):
            loss = torch.full_like(want[0], math.nan)
            dh = torch.full_like(want[1], math.nan) if which == 1 else None
            dt = torch.full_like(want[2], math.nan) if which == 2 else None
            E.ecc_cross_entropy(a, loss, dh, D, dt, D, V * D, 0, work, stream)
            assert torch.equal(loss, want[0])
            assert torch.equal(*((dh, want[1]) if which == 1 else (dt, want[2])))


def test_single_rows_and_far_rows():
    """A vector and its label, and rows further apart than 32 bits reach."""
    lm = _lm()
    announce("cross entropy, single and far rows")
    for dtype in (BF16, F32):
        h, table, y, w = _inputs(40, 64, 150, dtype, 14)
        y.clamp_(0, 149)
        want = lm.cross_entropy(h[3], table, y[3])
        assert want[0].shape == () and want[1].shape == (64,)
        assert torch.equal(want[1], lm.cross_entropy(h[3:4], table, y[3:4])[1][0])
    h, table, y, w = _inputs(40, 64, 40, BF16, 15)
    want = lm.cross_entropy(h, table, y, w)
    pitch = (1 << 27) + 8
    far = torch.empty(40 * pitch, dtype=BF16, device="cuda").view(40, pitch)
    wide = [far[:, 64 * i:64 * (i + 1)] for i in range(4)]
    wide[0].copy_(h)
    wide[1].copy_(table)
    got = lm.cross_entropy(wide[0], wide[1], y, w, dh=wide[2], dtable=wide[3][None])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_alike_weights():
    """Weights that are all alike are a factor of the sums: a label's term, near
    the weight in every row of a model that knows nothing yet, is off by no
    common half step of bf16."""
    lm = _lm()
    announce("cross entropy, alike weights")
    N, D, V = 512, 128, 2000
    h, table, y, _ = _inputs(N, D, V, BF16, 16, size=0.1)
    y.random_(0, V, generator=torch.Generator(device="cuda").manual_seed(1))
    for value in (1.0 / 515, 0.37, 3.0):
        w = torch.full((N,), value, device="cuda")
        _, dh, dt = _check(h, table, y, w)
        want = _reference(h, table, y, w, 1.0, 1, BF16)
        for got, (exact, _) in ((dh, want[1]), (dt, want[2])):
            # rounding the result leaves 2^-8 / sqrt(3) at most, and the terms
            # that are not labels as much of a small share
            error = (got.double() - exact).norm() / exact.norm()
            assert error <= 2.0 ** -8 / math.sqrt(3) * 1.1, float(error)


def test_work_buffers():
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("cross entropy, work buffers")
    for dtype in (BF16, F32):
        h, table, y, w = _inputs(90, 100, 275, dtype, 11)
        want = lm.cross_entropy(h, table, y, w)
        work = torch.full((1 << 22,), math.nan, device="cuda")
        got = lm.cross_entropy(h, table, y, w, work=work[8:])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        work.fill_(math.nan)
        assert torch.equal(lm.cross_entropy(h, table, y, w, grad=None, work=work[4:])[0], want[0])
        for bad in (work[:4], work.cpu(), work[::2]):
            with pytest.raises(ValueError):
                lm.cross_entropy(h, table, y, w, work=bad)
        with pytest.raises(E.EccError):
            lm.cross_entropy(h, table, y, w, work=work[1:])


def test_refusals():
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("cross entropy refusals")
    h, table, y, w = _inputs(12, 16, 8, F32, 12)
    for args in ((h, table[:, :15], y), (h[:, :8], table, y), (h, table, y[:11]), (h, table[0], y),
                 (h.t(), table, y), (h, table, y.long()), (h, table, y, w.double()),
                 (h, table, y, w[:11]), (h, table, y.cpu()), (h.cpu(), table.cpu(), y.cpu())):
        with pytest.raises(ValueError):
            lm.cross_entropy(*args)
    for args in ((h.half(), table, y), (h.double(), table.double(), y), (h, table.bfloat16(), y)):
        with pytest.raises(TypeError):
            lm.cross_entropy(*args)
    for dtype in (F64, BF16):
        with pytest.raises(TypeError):
            lm.cross_entropy(h, table, y, dtype=dtype)
    d = torch.empty((1, 8, 16), device="cuda")
    for kw in (dict(P=5), dict(accumulate=True), dict(grad=None, dtable=d), dict(P=2, dtable=d),
               dict(dh=h[:11]), dict(loss=w.double()), dict(loss=w[:3])):
        with pytest.raises(ValueError):
            lm.cross_entropy(h, table, y, **kw)

    def status(call):
        with pytest.raises(E.EccError) as e:
            call()
        return e.value.status
    assert status(lambda: lm.cross_entropy(h, table, y, dh=h)) == E.ECC_ERR_ARG
    assert status(lambda: lm.cross_entropy(h, table, y, dtable=table[None])) == E.ECC_ERR_ARG
    assert status(lambda: lm.cross_entropy(h, table, y, w, loss=w)) == E.ECC_ERR_ARG
    assert status(lambda: lm.cross_entropy(h, table, y, scale=math.inf)) == E.ECC_ERR_ARG
    assert status(lambda: lm.cross_entropy(h, table, y, scale=math.nan)) == E.ECC_ERR_ARG
    both = torch.empty((20, 16), device="cuda")
    assert status(lambda: lm.cross_entropy(h, table, y, dh=both[:12], dtable=both[10:18][None])) == \
        E.ECC_ERR_ARG
