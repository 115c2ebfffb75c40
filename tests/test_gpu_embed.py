"""Token embedding through the library's calls: the scaled lookup and the
table's gradient by sorted tokens, against their definitions in 64 bits.

Tolerances.  u = 2^-24 for fp32 sums, 2^-53 for fp64; a bf16 result (8
significant bits) adds 2^-8 relative.  A lookup is one rounded product.  A
gradient of m tokens adds m numbers in some order and scales once: its error
is at most (m + 3) u * scale * sum |dy|, whatever the order."""
import math
from fractions import Fraction

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from gpu_common import announce                           # noqa: E402

pytestmark = pytest.mark.gpu

F64, F32, BF16 = torch.float64, torch.float32, torch.bfloat16
HALF_ULP = {F64: 2.0 ** -53, F32: 2.0 ** -24, BF16: 2.0 ** -8}


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


def _unit(*types):
    return 2.0 ** -53 if F64 in types else 2.0 ** -24


def _random(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g, dtype=F64).to(dtype)


def _tokens(n, lo, hi, seed, common=0.0):
    """n tokens in [lo, hi); a share `common` of them one token."""
    rng = np.random.default_rng(seed)
    t = rng.integers(lo, hi, n)
    t[rng.random(n) < common] = (lo + hi) // 2
    return torch.from_numpy(t)


# ---------------------------------------------------------------------------
# lookup
# ---------------------------------------------------------------------------

def _lookup_ref(table, ids, scale, row0):
    r = ids.reshape(-1).long() - row0
    held = (r >= 0) & (r < table.shape[0])
    y = table.double()[r.clamp(0, table.shape[0] - 1)] * scale
    return torch.where(held[:, None], y, torch.zeros((), dtype=F64)).view(*ids.shape, -1)


@pytest.mark.parametrize("tt", [F64, F32, BF16])
@pytest.mark.parametrize("ot", [F64, F32, BF16])
@pytest.mark.parametrize("n,V,D", [(1, 1, 1), (3, 7, 5), (64, 50, 64), (257, 129, 250),
                                   (33, 1000, 1023), (5, 11, 4104)])
def test_lookup(tt, ot, n, V, D):
    announce("lookup", tt, ot, n, V, D)
    table, ids = _random((V, D), tt, 1), _tokens(n, -2, V + 2, 2)
    got = _lm().embed_lookup(table.cuda(), ids.cuda(), scale=3.7, dtype=ot).cpu().double()
    ref = _lookup_ref(table, ids, 3.7, 0)
    assert torch.all((got - ref).abs() <= (2 * _unit(tt, ot) + HALF_ULP[ot]) * ref.abs())


def test_lookup_no_tokens_and_shapes():
    lm = _lm()
    announce("lookup, empty")
    table = _random((9, 6), F32, 3).cuda()
    assert lm.embed_lookup(table, torch.empty((0,), dtype=torch.int64, device="cuda")).shape == \
        (0, 6)
    ids = _tokens(24, 0, 9, 4).view(2, 3, 4).cuda()
    got = lm.embed_lookup(table, ids)
    assert got.shape == (2, 3, 4, 6) and torch.equal(got, table[ids])


@pytest.mark.parametrize("id_type", [torch.int32, torch.int64])
def test_lookup_part_of_a_table(id_type):
    """Tables split by rows: the parts' lookups add up to the whole's; tokens
    far outside any 32-bit range are outside."""
    lm = _lm()
    announce("lookup, parts", id_type)
    table = _random((100, 40), F32, 5).cuda()
    ids = _tokens(300, 0, 100, 6).to(id_type)
    whole = lm.embed_lookup(table, ids.cuda(), scale=2.0)
    parts = sum(lm.embed_lookup(table[lo:hi], ids.cuda(), scale=2.0, row0=lo)
                for lo, hi in ((0, 37), (37, 38), (38, 100)))
    assert torch.equal(whole, parts)
    far = torch.tensor([-1, -100, 2 ** 31 - 1, -2 ** 31], dtype=id_type)
    if id_type == torch.int64:
        far = torch.cat([far, torch.tensor([2 ** 32, 2 ** 63 - 1, -2 ** 63, 2 ** 32 + 5])])
    for row0 in (0, 3):
        assert not lm.embed_lookup(table, far.cuda(), row0=row0).any()


def test_lookup_strided_and_unaligned():
    """Rows inside wider buffers, starting at any element."""
    lm = _lm()
    for dt, D, off in [(BF16, 61, 1), (BF16, 64, 3), (F32, 33, 1), (F64, 17, 1)]:
        announce("lookup, strided", dt, D, off)
        wide = _random((50, D + 9), dt, 7).cuda()
        table = wide[:, off:off + D]
        out = torch.full((40, D + 5), 8.0, dtype=dt, device="cuda")
        ids = _tokens(40, 0, 50, 8).cuda()
        lm.embed_lookup(table, ids, out=out[:, 2:2 + D])
        assert torch.equal(out[:, 2:2 + D], table[ids])
        assert (out[:, :2] == 8).all() and (out[:, 2 + D:] == 8).all()


def test_lookup_special_values():
    """Infinities and NaN of a row arrive; those of other rows do not, and a
    token outside the table gives zeros whatever the table holds."""
    lm = _lm()
    announce("lookup, special values")
    table = torch.full((4, 19), float("nan"), dtype=BF16)
    table[1] = 2.0
    table[2] = float("inf")
    got = lm.embed_lookup(table.cuda(), torch.tensor([1, 2, -1, 0, 4]).cuda(), scale=0.5).cpu()
    assert (got[0] == 1).all() and torch.isinf(got[1]).all()
    assert (got[2] == 0).all() and torch.isnan(got[3]).all() and (got[4] == 0).all()


# ---------------------------------------------------------------------------
# index and gradient
# ---------------------------------------------------------------------------

def _index_ref(ids, V, P, row0):
    n = ids.numel() // P
    r = ids.reshape(-1).long() - row0
    held = (r >= 0) & (r < V)
    key = torch.arange(P * n) // max(n, 1) * (V + 1) + torch.where(held, r, V)
    key, order = torch.sort(key, stable=True)
    return key, torch.where(held[order], order, ~order)


@pytest.mark.parametrize("P,n,V", [(1, 1, 1), (1, 63, 5), (1, 1024, 300), (1, 1025, 70000),
                                   (1, 2049, 7), (1, 4097, 128000), (1, 8193, 255),
                                   (1, 16384, 65535), (1, 16385, 1000), (1, 70001, 128000),
                                   (3, 5000, 40), (33, 77, 511), (2, 20011, 300000),
                                   (5, 17000, 65536)])
def test_index(P, n, V):
    """Both sorts: one workgroup per worker, and digits over tiles."""
    announce("index", P, n, V)
    ids = _tokens(P * n, -3, V + 3, P + n, common=0.3)
    index = _lm().embed_index(ids.cuda(), V, P=P)
    N = P * n
    at = (4 * N + 15) // 16 * 16
    data = index.data.cpu()
    key, order = _index_ref(ids, V, P, 0)
    assert torch.equal(data[:4 * N].view(torch.int32).long(), key)
    assert torch.equal(data[at:at + 4 * N].view(torch.int32).long(), order)


def _grad_ref(ids, dy, V, P, scale, row0=0):
    """(gradient, its error scale, tokens of each row)."""
    n = ids.numel() // P
    r = ids.reshape(-1).long() - row0
    held = (r >= 0) & (r < V)
    rows = torch.arange(P * n) // max(n, 1) * V + r
    rows, dy = rows[held], dy.reshape(P * n, -1)[held].double()
    shape = (P * V, dy.shape[1])
    g = torch.zeros(shape, dtype=F64).index_add_(0, rows, dy)
    s = torch.zeros(shape, dtype=F64).index_add_(0, rows, dy.abs())
    m = torch.bincount(rows, minlength=P * V)
    return ((g * scale).view(P, V, -1), (s * abs(scale)).view(P, V, -1),
            m.view(P, V, 1).double())


def _check_grad(got, ref, mass, count, u, ulp, before=None):
    got = got.cpu().double()
    tol = (count + 3) * u * mass
    want = ref if before is None else before.double() + ref
    if before is not None:
        tol = tol + 2 * u * (before.double().abs() + mass)
    assert torch.all((got - want).abs() <= tol + ulp * want.abs()), (got - want).abs().max()


@pytest.mark.parametrize("yt,gt", [(BF16, F32), (BF16, F64), (BF16, BF16), (F32, F32),
                                   (F32, F64), (F32, BF16), (F64, F64), (F64, F32), (F64, BF16)])
@pytest.mark.parametrize("P,n,V,D,common", [
    (1, 1, 1, 1, 0.0), (1, 1, 5, 300, 0.0), (1, 7, 3, 17, 0.0), (2, 100, 40, 8, 0.5),
    (1, 1500, 30, 65, 0.9), (3, 333, 700, 250, 0.2), (1, 3000, 5000, 1030, 0.1)])
def test_grad(yt, gt, P, n, V, D, common):
    announce("grad", yt, gt, P, n, V, D, common)
    lm = _lm()
    ids, dy = _tokens(P * n, -1, V + 1, 3, common), _random((P * n, D), yt, 4)
    index = lm.embed_index(ids.cuda(), V, P=P)
    ref, mass, count = _grad_ref(ids, dy, V, P, 1.3)
    got = lm.embed_grad(index, dy.cuda(), scale=1.3, dtype=gt)
    assert got.shape == (P, V, D)
    _check_grad(got, ref, mass, count, _unit(yt, gt), HALF_ULP[gt])
    # the same bits again, and added to what is there
    before = _random((P, V, D), gt, 5)
    more = before.cuda()
    lm.embed_grad(index, dy.cuda(), scale=1.3, grad=more, accumulate=True)
    _check_grad(more, ref, mass, count, _unit(yt, gt), HALF_ULP[gt], before)
    assert torch.equal(got, lm.embed_grad(index, dy.cuda(), scale=1.3, dtype=gt))
    untouched = (count == 0).expand(P, V, D)
    assert torch.equal(more.cpu()[untouched], before[untouched])
    assert not got.cpu()[untouched].any()


@pytest.mark.parametrize("n,D", [(40000, 64), (40000, 520)])
def test_grad_long_runs(n, D):
    """One token makes up the whole text, or nearly: its pieces cover
    thousands of tiles."""
    lm = _lm()
    for common, V in ((1.0, 1), (0.97, 50)):
        announce("grad, long runs", n, D, common)
        ids, dy = _tokens(n, 0, V, 6, common), _random((n, D), BF16, 7)
        ref, mass, count = _grad_ref(ids, dy, V, 1, 1.0)
        got = lm.embed_grad(lm.embed_index(ids.cuda(), V), dy.cuda())
        _check_grad(got, ref, mass, count, 2.0 ** -24, 2.0 ** -24)


def test_grad_no_tokens():
    lm = _lm()
    announce("grad, no tokens")
    empty = torch.empty((0,), dtype=torch.int32, device="cuda")
    dy = torch.empty((0, 33), dtype=F32, device="cuda")
    got = torch.full((2, 10, 33), 5.0, device="cuda")
    index = lm.embed_index(empty, 10, P=2)
    lm.embed_grad(index, dy, grad=got, accumulate=True)
    assert (got == 5).all()
    lm.embed_grad(index, dy, grad=got)
    assert not got.any()
    # tokens, but none in the table: their rows are not read
    ids = torch.full((50,), -1, dtype=torch.int64, device="cuda")
    dy = torch.full((50, 33), float("nan"), device="cuda")
    assert not lm.embed_grad(lm.embed_index(ids, 10), dy).any()


def test_grad_nan_of_padding_stays_out():
    """NaN and infinities in rows of tokens outside the table, next to every
    other row."""
    lm = _lm()
    announce("grad, NaN in padding")
    n, V, D = 999, 20, 70
    ids, dy = _tokens(n, 0, V, 8), _random((n, D), F32, 9)
    ids[::3] = -1
    dy[::3] = float("nan")
    dy[::6] = float("inf")
    ref, mass, count = _grad_ref(ids, dy, V, 1, 1.0)
    got = lm.embed_grad(lm.embed_index(ids.cuda(), V), dy.cuda())
    _check_grad(got, ref, mass, count, 2.0 ** -24, 2.0 ** -24)


def test_grad_in_rank_contributions():
    """Workers' gradients inside the contributions of a stale allreduce: rows
    at their own stride, the elements around them left alone."""
    lm = _lm()
    announce("grad in contributions")
    P, n, V, D = 4, 120, 33, 31
    contrib = torch.full((P, 5 + V * (D + 2) + 3), 9.0, dtype=F64, device="cuda")
    view = contrib[:, 5:5 + V * (D + 2)].view(P, V, D + 2)[:, :, :D]
    ids, dy = _tokens(P * n, -1, V, 10), _random((P * n, D + 3), BF16, 11)
    ref, mass, count = _grad_ref(ids, dy[:, 1:1 + D], V, P, 0.25)
    lm.embed_grad(lm.embed_index(ids.cuda(), V, P=P), dy.cuda()[:, 1:1 + D], scale=0.25,
                  grad=view)
    _check_grad(view, ref, mass, count, 2.0 ** -53, 2.0 ** -53)
    rest = contrib.clone()
    rest[:, 5:5 + V * (D + 2)].view(P, V, D + 2)[:, :, :D] = 9.0
    assert (rest == 9).all()


def test_grad_of_part_of_a_table():
    lm = _lm()
    announce("grad of a table's part")
    n, V, D = 700, 90, 24
    ids, dy = _tokens(n, 0, V, 12), _random((n, D), F32, 13)
    ref, mass, count = _grad_ref(ids, dy, 40, 1, 1.0, row0=30)
    got = lm.embed_grad(lm.embed_index(ids.cuda(), 40, row0=30), dy.cuda())
    _check_grad(got, ref, mass, count, 2.0 ** -24, 2.0 ** -24)


def test_grad_against_differences():
    """The gradient of sum(lookup * c) in the table, against differences of
    the lookup in 64 bits (linear: exact but for rounding)."""
    lm = _lm()
    announce("grad against differences")
    n, V, D = 30, 6, 5
    ids, c = _tokens(n, -1, V, 14).cuda(), _random((n, D), F64, 15).cuda()
    table = _random((V, D), F64, 16).cuda()

    def value(t):
        return float((lm.embed_lookup(t, ids, scale=1.7) * c).sum())

    got = lm.embed_grad(lm.embed_index(ids, V), c, scale=1.7, dtype=F64)[0]
    for v in range(V):
        for d in range(D):
            up, down = table.clone(), table.clone()
            up[v, d] += 0.5
            down[v, d] -= 0.5
            assert abs(value(up) - value(down) - float(got[v, d])) <= 1e-12 * n * D


def test_on_another_stream():
    """Index and gradient on a stream of their own, joined by events."""
    lm = _lm()
    announce("another stream")
    n, V, D = 5000, 400, 96
    ids, dy = _tokens(n, 0, V, 17), _random((n, D), BF16, 18)
    d_ids, d_dy = ids.cuda(), dy.cuda()
    want = lm.embed_grad(lm.embed_index(d_ids, V), d_dy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = lm.embed_grad(lm.embed_index(d_ids, V), d_dy)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_in_a_graph():
    """Index, lookup and gradient captured once and replayed on new tokens."""
    lm = _lm()
    announce("graph")
    n, V, D = 3000, 500, 130
    ids, table = _tokens(n, -1, V, 19).cuda(), _random((V, D), F32, 20).cuda()
    dy = _random((n, D), F32, 21).cuda()
    lm.embed_grad(lm.embed_index(ids, V), lm.embed_lookup(table, ids))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = lm.embed_lookup(table, ids, scale=2.0)
        g = lm.embed_grad(lm.embed_index(ids, V), dy)
    for k in range(4):
        ids.copy_(_tokens(n, -1, V, 30 + k))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, lm.embed_lookup(table, ids, scale=2.0))
        assert torch.equal(g, lm.embed_grad(lm.embed_index(ids, V), dy))


def test_refusals():
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("embed refusals")
    table = torch.zeros((10, 8), device="cuda")
    ids = torch.zeros(6, dtype=torch.int64, device="cuda")
    out = torch.zeros((6, 8), device="cuda")

    def lookup(**kw):
        a = dict(n=6, V=10, D=8, row0=0, d_ids=ids, id_type=E.ECC_I64, d_table=table,
                 table_type=E.ECC_F32, ld_table=8, scale=1.0, d_out=out, out_type=E.ECC_F32,
                 ld_out=8)
        a.update(kw)
        with pytest.raises(E.EccError) as e:
            E.ecc_embed_lookup(**a)
        return e.value.status

    for bad in (dict(n=-1), dict(V=0), dict(D=0), dict(id_type=E.ECC_F32), dict(table_type=7),
                dict(out_type=E.ECC_I32), dict(ld_table=7), dict(ld_out=7), dict(d_ids=None),
                dict(d_table=None), dict(d_out=None), dict(d_out=table),
                dict(d_out=out.data_ptr() + 2), dict(d_ids=ids.data_ptr() + 4),
                dict(d_out=ids)):
        assert lookup(**bad) == E.ECC_ERR_ARG, bad
    assert lookup(V=1 << 33) == E.ECC_ERR_RANGE
    assert lookup(n=1 << 36) == E.ECC_ERR_RANGE

    index = lm.embed_index(ids, 10, P=2)
    work = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    grad = torch.zeros((2, 10, 8), device="cuda")

    def embed_grad(**kw):
        a = dict(P=2, n=3, V=10, D=8, d_index=index.data, d_dy=out, dy_type=E.ECC_F32, ld_dy=8,
                 scale=1.0, d_grad=grad, grad_type=E.ECC_F32, ld_grad=8, worker_stride=80,
                 accumulate=0, d_work=work)
        a.update(kw)
        with pytest.raises(E.EccError) as e:
            E.ecc_embed_grad(**a)
        return e.value.status

    for bad in (dict(P=0), dict(n=-1), dict(V=0), dict(D=0), dict(dy_type=E.ECC_I64),
                dict(grad_type=9), dict(ld_dy=7), dict(ld_grad=7), dict(worker_stride=79),
                dict(accumulate=2), dict(d_index=None), dict(d_dy=None), dict(d_grad=None),
                dict(d_work=None), dict(d_work=work.data_ptr() + 8),
                dict(d_index=index.data.data_ptr() + 4), dict(d_work=grad), dict(d_dy=grad),
                dict(d_grad=grad.data_ptr() + 1)):
        assert embed_grad(**bad) == E.ECC_ERR_ARG, bad
    assert embed_grad(n=1 << 31) == E.ECC_ERR_RANGE
    assert embed_grad(D=(1 << 22) + 1, ld_dy=1 << 23, ld_grad=1 << 23, worker_stride=1 << 27) == \
        E.ECC_ERR_RANGE
    with pytest.raises(E.EccError):
        E.ecc_embed_index(2, 3, 10, 0, ids, E.ECC_I64, index.data.data_ptr() + 4)
    with pytest.raises(E.EccError):
        E.ecc_embed_index(2, 3, 10, 0, None, E.ECC_I64, index.data)
    # what the tensors say
    with pytest.raises(TypeError):
        lm.embed_lookup(table, ids.float())
    with pytest.raises(TypeError):
        lm.embed_lookup(table.half(), ids)
    with pytest.raises(ValueError):
        lm.embed_lookup(table.t(), ids)
    with pytest.raises(ValueError):
        lm.embed_lookup(table, ids[::2])
    with pytest.raises(ValueError):
        lm.embed_lookup(table.cpu(), ids)
    with pytest.raises(ValueError):
        lm.embed_lookup(table, ids, out=out[:5])
    with pytest.raises(ValueError):
        lm.embed_index(ids, 10, P=4)
    with pytest.raises(ValueError):
        lm.embed_grad(index, out[:5])
    with pytest.raises(ValueError):
        lm.embed_grad(index, out, accumulate=True)
    with pytest.raises(ValueError):
        lm.embed_grad(index, out, grad=grad[:, :9])


def _bf16_bits(v):
    """bf16 nearest to the fp64 values v (ties to even), by whole numbers."""
    out = []
    for x in v.reshape(-1).tolist():
        m, e = math.frexp(abs(x))             # m in [0.5, 1)
        n = Fraction(m) * 256                 # 8 significant bits
        q = int(n)
        r = n - q
        q += r > Fraction(1, 2) or (r == Fraction(1, 2) and q % 2 == 1)
        out.append(math.copysign(math.ldexp(q, e - 8), x))
    return torch.tensor(out, dtype=F64).reshape(v.shape)


def test_fp64_is_rounded_to_bf16_once():
    """fp64 values next to the middle of two bf16 neighbours, nearer to it than
    fp32 resolves: rounded to the nearer neighbour, in the lookup and in the
    gradient, in whole accesses and at a row's end."""
    lm = _lm()
    announce("fp64 to bf16")
    g = torch.Generator().manual_seed(3)
    V, D = 40, 77
    middle = (torch.randint(128, 256, (V, D), generator=g, dtype=F64) + 0.5) * \
        2.0 ** torch.randint(-20, 20, (V, D), generator=g)
    off = (torch.randint(0, 3, (V, D), generator=g) - 1) * 2.0 ** -35
    sign = torch.randint(0, 2, (V, D), generator=g) * 2.0 - 1.0
    table = sign * middle * (1.0 + off)
    want = _bf16_bits(table)
    ids = torch.arange(V).cuda()
    got = lm.embed_lookup(table.cuda(), ids, dtype=BF16).cpu().double()
    assert torch.equal(got, want)
    index = lm.embed_index(ids, V)
    got = lm.embed_grad(index, table.cuda(), dtype=BF16)[0].cpu().double()
    assert torch.equal(got, want)
    inf, top, last = float("inf"), 2.0 ** 128 - 2.0 ** 120, 2.0 ** 128 - 2.0 ** 119
    special = torch.tensor([[inf, -inf, float("nan"), 0.0, -0.0, 1e300, -1e39,
                             math.nextafter(last, 0.0), last, 1e-300]], dtype=F64)
    got = lm.embed_lookup(special.cuda(), ids[:1], dtype=BF16).cpu().double()[0]
    assert got[:2].tolist() == [inf, -inf] and torch.isnan(got[2])
    assert got[3:].tolist() == [0.0, -0.0, inf, -inf, top, inf, 0.0] and \
        torch.signbit(got[4])


def test_work_buffers_that_do_not_hold():
    """Work buffers on the host, too small, or with fewer elements in memory than
    they show are refused, as are operands apart from each other."""
    lm = _lm()
    announce("embed, work buffers")
    ids, dy = torch.zeros(6, dtype=torch.int64, device="cuda"), torch.zeros((6, 8), device="cuda")
    index = lm.embed_index(ids, 5)

    def call(work):
        return lm.embed_grad(index, dy, work=work)
    size = 1 << 24
    for work in (torch.empty(size, dtype=torch.uint8), torch.empty(8, device="cuda")[:1],
                 torch.empty(1, dtype=torch.uint8, device="cuda").expand(size),
                 torch.empty(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            call(work)
    call(torch.empty(size, dtype=torch.uint8, device="cuda"))


def test_rows_beside_the_table():
    """Table, lookup and gradient as columns of one buffer."""
    from paper_2203_17063_amd import capi as E
    lm = _lm()
    announce("embed, rows beside each other")
    n, D = 30, 19
    wide = torch.full((n, 3 * D + 1), 5.0, device="cuda")
    table, out, grad = (wide[:, k * D:(k + 1) * D] for k in range(3))
    table.copy_(_random((n, D), F32, 1))
    ids = _tokens(n, 0, n, 2).cuda()
    lm.embed_lookup(table, ids, out=out)
    assert torch.equal(out, table[ids])
    index = lm.embed_index(ids, n)
    want = lm.embed_grad(index, out.clone())
    lm.embed_grad(index, out, grad=grad[None])
    assert torch.equal(grad, want[0]) and (wide[:, 3 * D] == 5).all()
    assert torch.equal(out, table[ids])
    for k in (D - 1, 1):
        with pytest.raises(E.EccError) as e:
            lm.embed_lookup(table, ids, out=wide[:, k:k + D])
        assert e.value.status == E.ECC_ERR_ARG
    with pytest.raises(E.EccError):
        lm.embed_grad(index, out, grad=wide[None, :, 2 * D - 1:3 * D - 1])


def test_lookup_of_more_than_one_launch():
    """An output of more than 32 GiB: more workgroups than one launch takes."""
    lm = _lm()
    n, V, D = (1 << 23) + 5, 300, 2048
    if torch.cuda.mem_get_info()[0] < 2 * n * D + (8 << 30):
        pytest.skip("not enough device memory")
    announce("lookup, 34 GB")
    table, ids = _random((V, D), BF16, 1).cuda(), torch.arange(n, device="cuda") % V
    out = torch.full((n, D), 7.0, dtype=BF16, device="cuda")
    lm.embed_lookup(table, ids, out=out)
    for lo in list(range(0, n, 1 << 20)) + [n - 1000]:
        hi = min(n, lo + 1000)
        assert torch.equal(out[lo:hi], table[ids[lo:hi]])
    at = torch.randint(0, n, (100000,), device="cuda")
    assert torch.equal(out[at], table[ids[at]])
    del out
    torch.cuda.empty_cache()


def test_index_of_many_workers():
    """Four million workers of two tokens and their gradients: more workgroups
    than one launch of fewer than 2^32 threads has."""
    lm = _lm()
    P, n, V = (1 << 22) + 3, 2, 3
    announce("index, many workers", P, n, V)
    ids = torch.randint(-1, V + 1, (P * n,), generator=torch.Generator().manual_seed(1))
    index = lm.embed_index(ids.cuda(), V, P=P)
    key, order = _index_ref(ids, V, P, 0)
    N = P * n
    at = (4 * N + 15) // 16 * 16
    data = index.data.cpu()
    assert torch.equal(data[:4 * N].view(torch.int32).long(), key)
    assert torch.equal(data[at:at + 4 * N].view(torch.int32).long(), order)
    dy = _random((N, 2), F32, 2)
    ref, mass, count = _grad_ref(ids, dy, V, P, 1.0)
    got = lm.embed_grad(index, dy.cuda())
    _check_grad(got, ref, mass, count, 2.0 ** -24, 2.0 ** -24)


def test_grad_of_more_than_128_gib():
    """A contiguous gradient of 137 GB, most of it zeros."""
    lm = _lm()
    V, D, n = (1 << 25) + 3, 1024, 1000
    if torch.cuda.mem_get_info()[0] < 4 * V * D + (8 << 30):
        pytest.skip("not enough device memory")
    announce("grad, 137 GB")
    ids = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(5))
    ids[0], ids[1], ids[2] = 0, V - 1, V - 1
    dy = torch.randn((n, D), device="cuda")
    grad = torch.empty((1, V, D), device="cuda")
    grad.fill_(3.0)
    index = lm.embed_index(ids.cuda(), V)
    lm.embed_grad(index, dy, grad=grad)
    rows, inverse = torch.unique(ids.cuda(), return_inverse=True)
    want = torch.zeros((rows.numel(), D), dtype=F64, device="cuda").index_add_(0, inverse,
                                                                             dy.double())
    assert (grad[0, rows].double() - want).abs().max() <= 1e-5
    # every other element is zero
    step = 1 << 21
    nonzero = sum(int(torch.count_nonzero(grad[0, lo:lo + step])) for lo in range(0, V, step))
    assert nonzero == int(torch.count_nonzero(grad[0, rows]))
    del grad
    torch.cuda.empty_cache()


def test_grad_of_many_rows():
    """P V beyond 2^29 rows."""
    lm = _lm()
    announce("grad, many rows")
    P, V, D, n = 2, (1 << 28) + 100, 1, 5000
    if torch.cuda.mem_get_info()[0] < (16 << 30):
        pytest.skip("not enough device memory")
    ids, dy = _tokens(P * n, 0, V, 3).cuda(), _random((P * n, D), F32, 4).cuda()
    ids[0], ids[n - 1], ids[-1] = 0, V - 1, V - 1
    grad = torch.full((P, V, D), 2.0, device="cuda")
    lm.embed_grad(lm.embed_index(ids, V, P=P), dy, grad=grad)
    rows = torch.arange(P * n, device="cuda") // n * V + ids
    want = torch.zeros(P * V, dtype=F64, device="cuda").index_add_(0, rows, dy[:, 0].double())
    assert (grad.view(-1).double() - want).abs().max() <= 1e-5


def _grad_on_device(ids, dy, V, cols):
    """The gradient's columns `cols` and their masses in 64 bits on the GPU, a
    token at a time off the sorted order."""
    r = ids.long()
    held = (r >= 0) & (r < V)
    y = dy[held][:, cols].double()
    zero = torch.zeros((V, len(cols)), dtype=F64, device="cuda")
    g, s = zero.clone(), zero
    order = torch.sort(r[held], stable=True)
    rows, count = torch.unique_consecutive(order.values, return_counts=True)
    for out, v in ((g, y), (s, y.abs())):
        c = torch.cumsum(v[order.indices], 0)[torch.cumsum(count, 0) - 1]
        out[rows] = torch.cat([c[:1], c[1:] - c[:-1]])
    m = torch.zeros((V, 1), dtype=F64, device="cuda")
    m[rows, 0] = count.double()
    return g, s, m


@pytest.mark.parametrize("n,D,tile,V,common", [
    (131072, 4096, 32, 3000, 0.3), (131071, 4103, 32, 100, 0.0), (262144, 4096, 64, 5000, 0.5),
    (262147, 4099, 64, 701, 0.01), (70001, 4096, 16, 997, 0.9), (131072, 8192, 64, 1, 0.0)])
def test_grad_longer_tiles(n, D, tile, V, common):
    """Sums over so many tokens that tiles hold 16, 32 and 64 of them: runs
    shorter than a tile, of its length and around it, of twice that, and of
    thousands of tiles, tokens outside the table in between."""
    lm = _lm()
    announce("grad, longer tiles", n, D, tile, V, common)
    rng = np.random.default_rng(n + D)
    t = rng.integers(0, V, n)
    t[rng.random(n) < common] = V // 2
    t[rng.random(n) < 0.02] = -1
    if V > 600:
        # runs of given lengths, at what place the others leave them
        at = 0
        for k, length in enumerate([tile - 1, tile, tile + 1, 2 * tile, 2 * tile - 1, 2 * tile + 1,
                                    1, 2, 3 * tile, 5] * 6):
            t[t == 10 + 3 * k] = V // 2
            t[at:at + length] = 10 + 3 * k
            at += length
    ids = torch.from_numpy(t).cuda()
    dy = torch.randn((n, D), dtype=BF16, device="cuda",
                     generator=torch.Generator(device="cuda").manual_seed(n))
    dy[ids < 0] = float("nan")
    grad = lm.embed_grad(lm.embed_index(ids, V), dy)[0]
    assert torch.isfinite(grad).all()
    cols = list(range(8)) + [500, 511, 512, 513, 1024, D // 2, D - 513, D - 512] + \
        list(range(D - 8, D))
    g, s, m = _grad_on_device(ids, dy, V, cols)
    # (the reference's running sums: a few units of 2^-53 of the whole column)
    tol = (m + 4) * 2.0 ** -24 * s + 1e-9
    assert ((grad[:, cols].double() - g).abs() <= tol).all()
    again = lm.embed_grad(lm.embed_index(ids, V), dy)[0]
    assert torch.equal(grad, again)


@pytest.mark.parametrize("gt,V,D,n", [
    (F32, 40000, 2048, 45000),     # above 256 MiB, few rows without tokens
    (F64, 9001, 4099, 9100),       # the same, rows of odd lengths
    (F32, 3000, 4096, 500),        # rows of 16 KiB
    (F32, 3001, 5120, 2000),       # of 20 KiB
    (F64, 1501, 3500, 900),        # of 28,000 bytes
    (F32, 40001, 4096, 30000),     # of 16 KiB, above 256 MiB
    (BF16, 1201, 16385, 700),      # of 32 KiB and two bytes
    (BF16, 33000, 10240, 25000),   # of 20 KiB, above 256 MiB
    (F32, 3001, 7000, 2500),       # of 28,000 bytes
    (F32, 15001, 6144, 10000),     # of 24 KiB, above 256 MiB
    (F32, 14999, 8191, 15000)])    # of 4 bytes less than 32 KiB, above 256 MiB
def test_grad_zeros(gt, V, D, n):
    """Rows without tokens in large gradients and in rows of 16 to 32 KiB: all
    of them zeros, the others complete."""
    lm = _lm()
    announce("grad, zeros", gt, V, D, n)
    yt = F32 if gt != BF16 else BF16
    ids = _tokens(n, -1, V, n).cuda()
    dy = torch.randn((n, D), dtype=yt, device="cuda",
                     generator=torch.Generator(device="cuda").manual_seed(n))
    grad = torch.full((1, V, D), float("nan"), dtype=gt, device="cuda")
    lm.embed_grad(lm.embed_index(ids, V), dy, grad=grad)
    touched = torch.zeros(V, dtype=torch.bool, device="cuda")
    touched[ids[ids >= 0]] = True
    assert torch.isfinite(grad).all() and not grad[0, ~touched].any()
    cols = [0, 1, 2, 3, D // 2, D - 3, D - 2, D - 1]
    g, s, m = _grad_on_device(ids, dy, V, cols)
    u = _unit(yt, gt)
    tol = (m + 4) * u * s + HALF_ULP[gt] * g.abs() + 1e-9
    assert ((grad[0][:, cols].double() - g).abs() <= tol).all()
