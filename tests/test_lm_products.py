"""Sizes and refusals of the feed-forward block, cross entropy from hidden
states and clipping that need no GPU: the size calls, and argument errors found
before anything is enqueued."""
import math

import pytest

from paper_2203_17063_amd import capi as E


def _ce(**kw):
    d = dict(n=100, V=1000, D=64, P=2, type=E.ECC_F32, grad_type=E.ECC_F32, pad=0, d_h=1 << 20,
             ld_h=64, d_table=2 << 20, ld_table=64, d_labels=3 << 20, d_weight=None, scale=1.0)
    d.update(kw)
    return E.ecc_cross_entropy_t(**d)


def _ffn(**kw):
    d = dict(n=100, D=64, F=200, P=2, type=E.ECC_F32, grad_type=E.ECC_F32, act=E.ECC_ACT_SILU,
             d_x=1 << 20, ld_x=64, d_w_gate=2 << 20, ld_gate=64, d_w_up=3 << 20, ld_up=64)
    d.update(kw)
    return E.ecc_ffn_t(**d)


def _tensors(*each):
    d = dict(d_grad=1 << 20, d_out=None, n=100, stride=100, out_stride=0, type=E.ECC_F32,
             out_type=0)
    return (E.ecc_tensor_t * len(each))(*[E.ecc_tensor_t(**dict(d, **e)) for e in each])


BF16 = dict(type=E.ECC_BF16, grad_type=E.ECC_BF16)


def test_cross_entropy_work_size():
    alone, both = (E.ecc_cross_entropy_work_size(_ce(), g) for g in (0, 1))
    # the table's pieces; rows' logits, and their gradients twice in three pieces
    assert alone >= 3 * 2 * 1000 * 64
    assert both >= alone + 2 * 128 * 1024 * 4 + 2 * 3 * 2 * 256 * 1000
    assert E.ecc_cross_entropy_work_size(_ce(n=0, d_h=None, d_labels=None), 1) >= 16
    # a bf16 table of whole, aligned rows is read as it lies
    lies, gap = (E.ecc_cross_entropy_work_size(_ce(ld_table=ld, **BF16), 0) for ld in (64, 66))
    assert gap >= lies + 2 * 1000 * 64
    # pieces of rows are bounded, however many there are
    big = [E.ecc_cross_entropy_work_size(_ce(n=n, V=128000, D=4096, ld_h=4096, ld_table=4096, P=1,
                                             **BF16), 1) for n in (1 << 14, 1 << 18)]
    table = 128000 * 4096
    # (the table transposed, its sums in fp32, parts of a split product)
    assert all(size < (5 << 30) + 2 * table + 4 * table + (1 << 30) for size in big)


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(V=0), dict(D=0), dict(P=0), dict(type=E.ECC_F64), dict(type=7),
    dict(grad_type=E.ECC_F64), dict(grad_type=E.ECC_BF16), dict(scale=math.inf),
    dict(scale=math.nan), dict(ld_h=63), dict(ld_table=63), dict(d_h=None), dict(d_table=None),
    dict(d_labels=None), dict(d_h=(1 << 20) + 2), dict(d_table=(1 << 20) + 1),
    dict(d_labels=(1 << 20) + 2), dict(d_weight=(1 << 20) + 2),
    dict(V=E.ECC_CROSS_ENTROPY_MAX_VOCAB + 1), dict(D=E.ECC_CROSS_ENTROPY_MAX_DIM + 1,
                                                    ld_h=1 << 17, ld_table=1 << 17),
    dict(n=1 << 31), dict(n=1, P=1 << 25), dict(ld_h=1 << 40), dict(ld_table=1 << 40),
    dict(V=1 << 22, D=1 << 15, ld_h=1 << 15, ld_table=1 << 15)])
def test_cross_entropy_refused(bad):
    a = _ce(**bad)
    assert E.ecc_cross_entropy_work_size(a, 1) == -1
    with pytest.raises(E.EccError) as e:
        E.ecc_cross_entropy(a, 4 << 20, None, 0, None, 0, 0, 0, 1 << 30)
    wide = any(k in bad for k in ("ld_h", "ld_table")) and bad.get("ld_h", 64) != 63 and \
        bad.get("ld_table", 64) != 63
    over = wide or bad.get("V", 0) > 1 << 21 or bad.get("n", 0) > 1 << 30 or \
        bad.get("P", 0) > 1 << 20
    assert e.value.status == (E.ECC_ERR_RANGE if over else E.ECC_ERR_ARG)
    assert E.ecc_last_error() != ""


@pytest.mark.parametrize("P", [1, 64])
def test_cross_entropy_rows(P):
    # (a launch has fewer than 2^32 threads, some of them 64 for each row)
    most = E.ECC_CROSS_ENTROPY_MAX_ROWS // P
    assert E.ecc_cross_entropy_work_size(_ce(P=P, n=most, V=3, D=1), 1) > 20 * most * P
    a = _ce(P=P, n=most + 1, V=3, D=1)
    assert E.ecc_cross_entropy_work_size(a, 1) == -1
    with pytest.raises(E.EccError) as e:
        E.ecc_cross_entropy(a, 4 << 20, None, 0, None, 0, 0, 0, 1 << 30)
    assert e.value.status == E.ECC_ERR_RANGE


def test_cross_entropy_outputs_refused():
    a, work = _ce(), 1 << 32
    good = dict(d_loss=4 << 20, d_dh=5 << 20, ld_dh=64, d_dtable=6 << 20, ld_dtable=64,
                worker_stride=64000, accumulate=0, d_work=work)
    for bad in (dict(d_loss=None), dict(d_work=None), dict(d_loss=(4 << 20) + 2),
                dict(d_dh=(5 << 20) + 2), dict(d_work=work + 8), dict(ld_dh=63),
                dict(ld_dtable=63), dict(worker_stride=63999), dict(accumulate=2),
                dict(accumulate=-1), dict(d_dh=1 << 20), dict(d_dtable=2 << 20),
                dict(d_loss=(3 << 20) + 64), dict(d_loss=5 << 20),
                dict(d_dtable=(5 << 20) + 128), dict(d_work=6 << 20)):
        with pytest.raises(E.EccError) as e:
            E.ecc_cross_entropy(a, **dict(good, **bad))
        assert e.value.status == E.ECC_ERR_ARG, bad
    for bad in (dict(ld_dh=1 << 40), dict(ld_dtable=1 << 36, worker_stride=1 << 50),
                dict(worker_stride=1 << 56)):
        with pytest.raises(E.EccError) as e:
            E.ecc_cross_entropy(a, **dict(good, **bad))
        assert e.value.status == E.ECC_ERR_RANGE, bad


def test_ffn_work_size():
    forward, grad = (E.ecc_ffn_work_size(_ffn(), g) for g in (0, 1))
    assert forward >= 3 * 2 * (200 + 2 * 200) * 64
    # dg and du in both orders, three pieces
    assert grad >= forward + 2 * 3 * 2 * 200 * 2 * 200
    # bf16 operands of whole, aligned rows are read as they lie
    assert E.ecc_ffn_work_size(_ffn(**BF16), 0) == 16
    assert E.ecc_ffn_work_size(_ffn(ld_up=72, **BF16), 0) >= 2 * 2 * 200 * 64
    assert E.ecc_ffn_work_size(_ffn(d_x=(1 << 20) + 2, **BF16), 0) >= 2 * 200 * 64
    assert E.ecc_ffn_work_size(_ffn(n=0, d_x=None, d_w_gate=None, d_w_up=None), 1) >= 16


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(D=0), dict(F=0), dict(P=0), dict(type=E.ECC_F64), dict(grad_type=E.ECC_F64),
    dict(grad_type=E.ECC_BF16), dict(act=2), dict(act=-1), dict(ld_x=63), dict(ld_gate=63),
    dict(ld_up=63), dict(d_x=None), dict(d_w_gate=None), dict(d_w_up=None),
    dict(d_x=(1 << 20) + 2), dict(d_w_up=(1 << 20) + 1)])
def test_ffn_refused(bad):
    a = _ffn(**bad)
    assert E.ecc_ffn_work_size(a, 0) == -1
    for call in (lambda: E.ecc_ffn_forward(a, 4 << 20, 200, 1 << 30),
                 lambda: E.ecc_ffn_grad(a, 4 << 20, 200, 5 << 20, 64, None, None, 0, 0, 1 << 30)):
        with pytest.raises(E.EccError) as e:
            call()
        assert e.value.status == E.ECC_ERR_ARG


@pytest.mark.parametrize("bad", [
    dict(n=E.ECC_FFN_MAX_ROWS + 1), dict(n=1, P=1 << 17), dict(F=E.ECC_FFN_MAX_DIM + 1),
    dict(D=E.ECC_FFN_MAX_DIM + 1, ld_x=1 << 21, ld_gate=1 << 21, ld_up=1 << 21),
    dict(ld_x=1 << 40), dict(ld_gate=1 << 40), dict(ld_up=1 << 40),
    dict(n=1 << 20, F=1 << 20), dict(P=1 << 14, n=1, F=1 << 19)])
def test_ffn_out_of_range(bad):
    a = _ffn(**bad)
    assert E.ecc_ffn_work_size(a, 0) == -1
    with pytest.raises(E.EccError) as e:
        E.ecc_ffn_forward(a, 4 << 20, 1 << 21, 1 << 30)
    assert e.value.status == E.ECC_ERR_RANGE


def test_ffn_outputs_refused():
    a, work = _ffn(), 1 << 32
    for y, ld, w in ((None, 200, work), (4 << 20, 199, work), (4 << 20, 200, None),
                     ((4 << 20) + 2, 200, work), (4 << 20, 200, work + 8), (1 << 20, 200, work),
                     ((2 << 20) - 800, 200, work), (4 << 20, 200, 4 << 20), (4 << 20, 200, 3 << 20)):
        with pytest.raises(E.EccError) as e:
            E.ecc_ffn_forward(a, y, ld, w)
        assert e.value.status == E.ECC_ERR_ARG, (y, ld, w)
    good = dict(d_dy=4 << 20, ld_dy=200, d_dx=5 << 20, ld_dx=64, d_dw_gate=6 << 20,
                d_dw_up=7 << 20, worker_stride=12800, accumulate=0, d_work=work)
    for bad in (dict(d_dy=None), dict(ld_dy=199), dict(ld_dx=63), dict(d_dw_gate=None),
                dict(d_dw_up=None), dict(worker_stride=12799), dict(accumulate=3),
                dict(d_work=None), dict(d_dy=(4 << 20) + 2), dict(d_dx=(5 << 20) + 1),
                dict(d_dw_up=(7 << 20) + 2), dict(d_work=work + 4), dict(d_dx=1 << 20),
                dict(d_dx=4 << 20), dict(d_dw_gate=2 << 20), dict(d_dw_up=6 << 20),
                dict(d_dw_up=(6 << 20) + 51200 - 4), dict(d_work=7 << 20)):
        with pytest.raises(E.EccError) as e:
            E.ecc_ffn_grad(a, **dict(good, **bad))
        assert e.value.status == E.ECC_ERR_ARG, bad
    for bad in (dict(ld_dy=1 << 40), dict(ld_dx=1 << 40), dict(worker_stride=1 << 56)):
        with pytest.raises(E.EccError) as e:
            E.ecc_ffn_grad(a, **dict(good, **bad))
        assert e.value.status == E.ECC_ERR_RANGE, bad


def test_norm_work_size():
    few = E.ecc_grad_norm_work_size(2, 1, _tensors({}))
    assert few >= 2 * 8
    many = E.ecc_grad_norm_work_size(2, 100, _tensors(*[{}] * 100))
    assert many >= 100 * (2 * 8 + 48)
    assert E.ecc_grad_norm_work_size(1, 0, None) >= 16
    # sums of chunks: of a bounded number, whatever the length
    assert E.ecc_grad_norm_work_size(1, 1, _tensors(dict(n=1 << 36))) < 1 << 20


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(type=E.ECC_I32), dict(type=-1), dict(d_grad=None), dict(d_grad=(1 << 20) + 2),
    dict(stride=99)])
def test_norm_refused(bad):
    t = _tensors({}, dict(d_grad=2 << 20, **{k: v for k, v in bad.items() if k != "d_grad"})
                 if "d_grad" not in bad else bad)
    assert E.ecc_grad_norm_work_size(2, 2, t) == -1
    for call in (lambda: E.ecc_grad_norm(2, 2, t, 4 << 20, 5 << 20),
                 lambda: E.ecc_clip_grads(2, 2, t, 1.0, E.ECC_CLIP_KEEP, 4 << 20, 5 << 20)):
        with pytest.raises(E.EccError) as e:
            call()
        assert e.value.status == E.ECC_ERR_ARG


def test_clip_refused():
    def status(tensors, P=2, limit=1.0, nonfinite=E.ECC_CLIP_KEEP, norms=8 << 20, work=9 << 20):
        with pytest.raises(E.EccError) as e:
            E.ecc_clip_grads(P, len(tensors), _tensors(*tensors), limit, nonfinite, norms, work)
        return e.value.status
    for kw in (dict(P=0), dict(limit=-1.0), dict(limit=math.nan), dict(nonfinite=2),
               dict(nonfinite=-1), dict(norms=None), dict(work=None), dict(norms=(8 << 20) + 4),
               dict(work=(9 << 20) + 8), dict(norms=1 << 20), dict(work=1 << 20),
               dict(work=8 << 20)):
        assert status([{}], **kw) == E.ECC_ERR_ARG, kw
    assert status([{}], P=65536) == E.ECC_ERR_RANGE
    assert status([dict(n=1 << 45, stride=1 << 45)]) == E.ECC_ERR_RANGE
    assert status([dict(stride=1 << 56)]) == E.ECC_ERR_RANGE
    out = dict(d_out=4 << 20, out_stride=100, out_type=E.ECC_F32)
    assert status([dict(out, out_stride=1 << 56)]) == E.ECC_ERR_RANGE
    for bad in (dict(out_type=9), dict(out_stride=99), dict(d_out=(4 << 20) + 2),
                dict(d_out=(1 << 20) + 4), dict(d_out=1 << 20, out_type=E.ECC_BF16),
                dict(d_out=1 << 20, out_stride=101), dict(d_out=8 << 20), dict(d_out=9 << 20)):
        assert status([dict(out, **bad)]) == E.ECC_ERR_ARG, bad
    other = dict(d_grad=2 << 20)
    for pair in ([out, dict(other, **out)], [dict(out, d_out=2 << 20), other], [{}, {}],
                 # rows of one pitch, one element over each other, the later one first
                 [dict(out, out_stride=400), dict(other, **dict(out, out_stride=400,
                                                               d_out=(4 << 20) + 396))],
                 [dict(other, **dict(out, out_stride=400, d_out=(4 << 20) + 396)),
                  dict(out, out_stride=400)]):
        assert status(pair) == E.ECC_ERR_ARG, pair
    with pytest.raises(E.EccError) as e:
        E.ecc_grad_norm(1, 1, _tensors({}), 1 << 20, 9 << 20)
    assert e.value.status == E.ECC_ERR_ARG


@pytest.mark.parametrize("wide_grad", [False, True])
@pytest.mark.parametrize("wide_out", [False, True])
@pytest.mark.parametrize("P", [None, 1, 3])
def test_workers_of_gradients_and_outputs(wide_grad, wide_out, P, monkeypatch):
    """What the library is told of dense gradients and of gradients within wider
    buffers, beside dense outputs and outputs within wider ones: a worker's
    elements, and each tensor's own distance from one worker to the next."""
    torch = pytest.importorskip("torch")
    from paper_2203_17063_amd import lm
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0, raising=False)
    lead = () if P is None else (P,)

    def tensors(wide, pitch, dtype):
        if P is None or not wide:
            return [torch.zeros(lead + s, dtype=dtype) for s in ((2, 5), (7,))]
        flat = torch.zeros((P, pitch), dtype=dtype)
        return [flat[:, 3:13].unflatten(1, (2, 5)), flat[:, 20:27]]
    grads, outs = tensors(wide_grad, 100, torch.float32), tensors(wide_out, 60, torch.float64)
    a, first = lm._tensors(grads, outs, P)
    assert first is grads[0] and len(a) == 2
    for t, g, o, n in zip(a, grads, outs, (10, 7)):
        assert (t.d_grad, t.d_out, t.n) == (g.data_ptr(), o.data_ptr(), n)
        assert (t.type, t.out_type) == (E.ECC_F32, E.ECC_F64)
        if P == 3:    # (of one worker there is no distance)
            assert t.stride == (100 if wide_grad else n)
            assert t.out_stride == (60 if wide_out else n)
    # the last worker's elements lie within the tensors that were given
    for t, g, o in zip(a, grads, outs):
        for at, stride, held in ((t.d_grad, t.stride, g), (t.d_out, t.out_stride, o)):
            memory = held.untyped_storage()
            end = at + (((P or 1) - 1) * stride + t.n) * held.element_size()
            assert end <= memory.data_ptr() + memory.nbytes()


@pytest.mark.parametrize("V", [1 << 20, 2000001, E.ECC_CROSS_ENTROPY_MAX_VOCAB])
@pytest.mark.parametrize("kinds", [(E.ECC_F32, E.ECC_F32), (E.ECC_BF16, E.ECC_F32),
                                   (E.ECC_BF16, E.ECC_BF16)])
def test_cross_entropy_pieces_of_large_vocabularies(V, kinds):
    """A piece's logits and gradients stay within 5 GiB, or 256 rows of them,
    however many rows there are."""
    operands, grads = (3 if kind == E.ECC_F32 else 1 for kind in kinds)
    # a logit in fp32, its gradient's pieces in both orders, 8 bytes for 64 of them
    row = (V + 63) // 64 * (64 * (4 + 2 * operands + 2 * grads) + 8)
    for P, n in ((1, 4096), (3, 100), (1, 1 << 20)):
        a = _ce(n=n, V=V, P=P, d_table=1 << 33, type=kinds[0], grad_type=kinds[1])
        # beside it: the table's pieces in both orders, sums of a bf16 gradient over
        # pieces of rows, and what is kept per row and worker
        rest = (2 * operands * 2 * 64 + 4 * P * 64) * (V + 64) + 64 * n * P + (1 << 26)
        assert E.ecc_cross_entropy_work_size(a, 1) < max(5 << 30, 256 * row) + rest
