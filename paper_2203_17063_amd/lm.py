"""Operators of language models over the C ABI: shapes, types and strides are
read from torch tensors and checked, outputs and work buffers allocated, and
libecc called on the current stream.  No arithmetic runs here.

The calls are not recorded for torch's differentiation: results of inputs that
require gradients do not, and the gradients are the calls named *_grad (and
distill's second result).

Rows (tokens, positions) may come with any number of leading dimensions as
long as the last one is contiguous and the others collapse to rows of one
stride.  Operands, outputs and work buffers of a call lie on one GPU, which
need not be the current one.  Sums over rows and tokens are held in fp32, or
fp64 where an operand or the result is fp64; a row's own sums (norms, softmax
statistics) in fp32, or fp64 for rows of fp64.
"""
from __future__ import annotations

import torch

from . import capi as E

_TYPES = {torch.float64: E.ECC_F64, torch.float32: E.ECC_F32, torch.bfloat16: E.ECC_BF16}
_ID_TYPES = {torch.int32: E.ECC_I32, torch.int64: E.ECC_I64}


# A device's current stream without the object around it (2.5 us of a call of
# 10), and the current device, where torch has them.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _launch(like, call, *args):
    """call(*args, stream), enqueued on the current stream of like's device,
    which is the current device meanwhile."""
    device = like.get_device()
    if device == _current_device():
        call(*args, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            call(*args, _raw_stream(device))


def _one_gpu(first, others, names):
    """`first` lies on a GPU, and the others (those that are not None) with it."""
    device = first.get_device()
    if device < 0:
        raise ValueError("%s must be on the GPU" % names.split()[0])
    for t in others:
        if t is not None and t.get_device() != device:
            what = names.split()[1 + [t is o for o in others].index(True)]
            raise ValueError("%s must be on %s, not on %s" % (what, first.device, t.device))


def _type(t, what):
    try:
        return _TYPES[t if isinstance(t, torch.dtype) else t.dtype]
    except KeyError:
        raise TypeError("%s must be float64, float32 or bfloat16, not %s" %
                        (what, t if isinstance(t, torch.dtype) else t.dtype)) from None


def _rows(t, what, cols=None):
    """(rows, leading dimension) of a tensor seen as a matrix of its last
    dimension."""
    d = t.dim()
    if d < 1 or (cols is not None and t.shape[-1] != cols):
        raise ValueError("%s must have %s in its last dimension, not shape %s" %
                         (what, "elements" if cols is None else cols, tuple(t.shape)))
    if t.is_contiguous():
        return (t.numel() // t.shape[-1] if t.shape[-1] else 0), t.shape[-1]
    if t.numel() and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError("%s must be contiguous in its last dimension" % what)
    if d == 1:
        return 1, t.shape[-1]
    m = t.view(-1, t.shape[-1]) if d > 2 else t   # (a view, or torch says why not)
    return m.shape[0], (m.stride(0) if m.shape[0] > 1 else m.shape[1])


def _contiguous(t, what):
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % what)
    return t


def _out(t, shape, dtype, like, what):
    """The caller's output, checked, or a new one where `like` is."""
    if t is None:
        return like.new_empty(shape, dtype=dtype)
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError("%s must be %s of shape %s, not %s of %s" %
                         (what, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    return t


def _work(size, like):
    if size < 0:
        raise E.EccError(E.ECC_ERR_RANGE, "the sizes are beyond what the library supports")
    return like.new_empty(size, dtype=torch.uint8)


def _given_work(work, size, like):
    """The caller's work buffer, checked."""
    _one_gpu(like, (_contiguous(work, "the work buffer"),), "- work")
    if work.numel() * work.element_size() < size:
        raise ValueError("the work buffer is too small")
    return work


# ----------------------------------------------------------------------------
# token embedding
# ----------------------------------------------------------------------------

def _ids(ids):
    if ids.dtype not in _ID_TYPES:
        raise TypeError("ids must be int32 or int64, not %s" % ids.dtype)
    return _contiguous(ids, "ids"), _ID_TYPES[ids.dtype]


def embed_lookup(table, ids, scale=1.0, dtype=None, out=None, row0=0):
    """scale * table[ids - row0], of shape ids.shape + (D,); zeros for tokens
    outside the table.  dtype: of the result (the table's by default)."""
    if table.dim() != 2:
        raise ValueError("table must be a matrix")
    V, D = table.shape
    tt = _type(table, "table")
    rows, ld = _rows(table, "table")
    ids, id_type = _ids(ids)
    dtype = out.dtype if out is not None else dtype or table.dtype
    ot = _type(dtype, "the result")
    out = _out(out, tuple(ids.shape) + (D,), dtype, table, "out")
    _, ld_out = _rows(out, "out")
    _one_gpu(table, (ids, out), "table ids out")
    _launch(table, E.ecc_embed_lookup, ids.numel(), V, D, row0, ids, id_type, table, tt, ld,
            scale, out, ot, ld_out)
    return out


class EmbedIndex:
    """The tokens of P workers sorted for embed_grad: P, tokens per worker n,
    table rows V, and the index's memory."""

    __slots__ = ("P", "n", "V", "data")

    def __init__(self, P, n, V, data):
        self.P, self.n, self.V, self.data = P, n, V, data


def embed_index(ids, V, P=1, row0=0, index=None):
    """Sorts the tokens of P workers (an equal share of ids each, worker after
    worker).  index: one of the same sizes whose memory is used again."""
    ids, id_type = _ids(ids)
    N = ids.numel()
    if P < 1 or N % P:
        raise ValueError("%d tokens cannot be shared equally by %d workers" % (N, P))
    n = N // P
    if index is None:
        index = EmbedIndex(P, n, V, _work(E.ecc_embed_index_size(P, n, V), ids))
    elif (index.P, index.n, index.V) != (P, n, V):
        raise ValueError("the index was made for other sizes")
    _one_gpu(ids, (index.data,), "ids index")
    _launch(ids, E.ecc_embed_index, P, n, V, row0, ids, id_type, index.data)
    return index


def embed_grad(index, dy, scale=1.0, grad=None, dtype=torch.float32, accumulate=False,
               work=None):
    """The table's gradient per worker, of shape (P, V, D): scale times the sum
    of the rows dy of each row's tokens.  grad: written, or with accumulate
    added to; its rows and workers may be strided."""
    P, n, V = index.P, index.n, index.V
    if dy.dim() < 1:
        raise ValueError("dy must have rows")
    D = dy.shape[-1]
    rows, ld_dy = _rows(dy, "dy")
    if rows != P * n:
        raise ValueError("dy has %d rows for %d tokens" % (rows, P * n))
    if grad is None:
        if accumulate:
            raise ValueError("accumulate needs grad")
        grad = index.data.new_empty((P, V, D), dtype=dtype)
    elif tuple(grad.shape) != (P, V, D):
        raise ValueError("grad must have shape %s, not %s" % ((P, V, D), tuple(grad.shape)))
    if D > 1 and grad.stride(2) != 1:
        raise ValueError("grad must be contiguous in its last dimension")
    _one_gpu(grad, (dy, index.data), "grad dy index")
    yt, gt = _type(dy, "dy"), _type(grad, "grad")
    size = E.ecc_embed_work_size(P, n, D, yt, gt)
    work = _work(size, grad) if work is None else _given_work(work, size, grad)
    _launch(grad, E.ecc_embed_grad, P, n, V, D, index.data, dy, yt, ld_dy, scale, grad, gt,
            grad.stride(1) if V > 1 else D, grad.stride(0) if P > 1 else V * D,
            1 if accumulate else 0, work)
    return grad


# ----------------------------------------------------------------------------
# norms, gate and residual around a block
# ----------------------------------------------------------------------------

def _vector(t, D, dtype, what):
    if t is None:
        return None
    if t.dim() != 1 or t.shape[0] != D or t.dtype != dtype:
        raise ValueError("%s must be %d elements of %s, not %s of %s" %
                         (what, D, dtype, tuple(t.shape), t.dtype))
    _contiguous(t, what)
    return t.data_ptr()


def _norm(x, f, w_post, w_pre, gate, gate_rows, res_scale, branch_scale, eps, offset, P):
    """The ecc_norm_t of tensors; rows and width."""
    D = x.shape[-1] if x.dim() else 0
    N, ld_x = _rows(x, "x")
    t = _type(x, "x")
    ld_f = 0
    if f is not None:
        rows, ld_f = _rows(f, "f", D)
        if rows != N or f.dtype != x.dtype:
            raise ValueError("f must be like x, not %s of shape %s" % (f.dtype, tuple(f.shape)))
    if P < 1 or N % P:
        raise ValueError("%d rows cannot be shared equally by %d workers" % (N, P))
    weights = [w for w in (w_post, w_pre, gate if gate is not None and gate_rows == 0 else None)
               if w is not None]
    w_dtype = weights[0].dtype if weights else x.dtype
    if gate_rows < 0:
        raise ValueError("gate_rows must be >= 0")
    ld_gate, d_gate = 0, None
    if gate is None:
        gate_rows = 0
    elif gate_rows == 0:
        d_gate = _vector(gate, D, w_dtype, "gate")
    else:
        rows, ld_gate = _rows(gate, "gate", D)
        if rows != -(-N // gate_rows) or gate.dtype != x.dtype:
            raise ValueError("gate must have %d rows of %s, not %s of %s" %
                             (-(-N // gate_rows), x.dtype, tuple(gate.shape), gate.dtype))
        d_gate = gate.data_ptr()
    a = E.ecc_norm_t(N // P, D, P, t, _type(w_dtype, "the weights"), x.data_ptr(), ld_x,
                     None if f is None else f.data_ptr(), ld_f, d_gate, ld_gate, gate_rows,
                     _vector(w_post, D, w_dtype, "w_post"), _vector(w_pre, D, w_dtype, "w_pre"),
                     offset, res_scale, branch_scale, eps)
    return a, N, D, w_dtype


def norm_forward(x, f=None, *, w_post=None, w_pre=None, gate=None, gate_rows=1, res_scale=1.0,
                 branch_scale=1.0, eps=1e-6, offset=0.0, x_out=None, h=None):
    """(x', h):  x' = res_scale x + branch_scale gate rms(f) (offset + w_post),
    h = rms(x') (offset + w_pre).

    Without w_post the branch is f itself, without f there is no branch and x'
    is None unless x_out is given or res_scale differs from 1; without w_pre h
    is None.  gate: rows like x's, each shared by gate_rows rows, or with
    gate_rows = 0 a parameter of x.shape[-1] elements.  x_out may be x, and h
    may be f."""
    a, N, D, _ = _norm(x, f, w_post, w_pre, gate, gate_rows, res_scale, branch_scale, eps, offset,
                       1)
    ld_xo = ld_h = 0
    if x_out is not None or f is not None or res_scale != 1.0 or w_pre is None:
        x_out = _out(x_out, x.shape, x.dtype, x, "x_out")
        _, ld_xo = _rows(x_out, "x_out")
    if w_pre is not None:
        h = _out(h, x.shape, x.dtype, x, "h")
        _, ld_h = _rows(h, "h")
    elif h is not None:
        raise ValueError("h needs w_pre")
    _one_gpu(x, (f, w_post, w_pre, gate, x_out, h), "x f w_post w_pre gate x_out h")
    _launch(x, E.ecc_norm_forward, a, x_out, ld_xo, h, ld_h)
    return x_out, h


def norm_grad(x, f=None, dh=None, dx_out=None, *, w_post=None, w_pre=None, gate=None, gate_rows=1,
              res_scale=1.0, branch_scale=1.0, eps=1e-6, offset=0.0, P=1, dtype=None, dx=None,
              df=None, dgate=None, dw_post=None, dw_pre=None, accumulate=False, work=None):
    """The gradients at x = x' of norm_forward, given those of h (dh) and of x'
    (dx_out, None for zero): a dict of dx, df, dgate, dw_post and dw_pre (None
    where the operand is absent).

    Parameters' gradients are per worker, (P, D) of dtype (the weights' type by
    default); given ones may be views of contributions whose rows lie one
    common stride apart, and accumulate adds to them.  dx may be dx_out or dh,
    df may be f or dh."""
    a, N, D, w_dtype = _norm(x, f, w_post, w_pre, gate, gate_rows, res_scale, branch_scale, eps,
                             offset, P)
    for t, of, what in ((df, f, "df"), (dgate, gate, "dgate"), (dw_post, w_post, "dw_post"),
                        (dw_pre, w_pre, "dw_pre")):
        if t is not None and of is None:
            raise ValueError("%s given without its operand" % what)
    wanted = [t for t, of in ((dw_post, w_post), (dw_pre, w_pre),
                              (dgate, gate if gate_rows == 0 else None)) if of is not None]
    given = [t for t in wanted if t is not None]
    dtype = given[0].dtype if given else dtype or w_dtype
    stride = given[0].stride(0) if given and P > 1 else D
    # new ones beside given ones in wide contributions are dense, and so are
    # those that the kernels write: the given ones are copies of them
    apart = stride != D and len(given) < len(wanted)
    copies = []

    def rows_in(t, what):
        if t is None:
            return None, 0
        rows, ld = _rows(t, what, D)
        if rows != N or t.dtype != x.dtype:
            raise ValueError("%s must be like x, not %s of shape %s" %
                             (what, t.dtype, tuple(t.shape)))
        return t.data_ptr(), ld

    def rows_out(t, like, what):
        if t is None:
            t = torch.empty_like(like, memory_format=torch.contiguous_format)
            return t, t.data_ptr(), D
        _out(t, like.shape, like.dtype, like, what)
        _, ld = _rows(t, what)
        return t, t.data_ptr(), ld

    def param(t, what):
        if t is None:
            if accumulate:
                raise ValueError("accumulate needs %s" % what)
            t = x.new_empty((P, D), dtype=dtype)
            return t, t.data_ptr()
        if tuple(t.shape) != (P, D) or t.dtype != dtype or (D > 1 and t.stride(1) != 1) or \
                (P > 1 and t.stride(0) != stride):
            raise ValueError("%s must be %s of shape %s, one stride for all" %
                             (what, dtype, (P, D)))
        if not apart:
            return t, t.data_ptr()
        if stride < D:
            raise ValueError("workers' gradients overlap")
        for other, _ in copies:   # (of the others the library sees where they are)
            at = (t.data_ptr() - other.data_ptr()) // t.element_size()
            if abs(at) < P * stride and min(at % stride, -at % stride) < D:
                raise ValueError("two gradients overlap")
        copies.append((t, t.new_empty((P, D))))
        return t, copies[-1][1].data_ptr()

    d_dh, ld_dh = rows_in(dh, "dh")
    d_dxo, ld_dxo = rows_in(dx_out, "dx_out")
    dx, d_dx, ld_dx = rows_out(dx, x, "dx")
    d_df = d_dgate = d_post = d_pre = None
    ld_df = ld_dgate = 0
    if f is not None:
        df, d_df, ld_df = rows_out(df, f, "df")
    if gate is not None:
        if gate_rows:
            dgate, d_dgate, ld_dgate = rows_out(dgate, gate, "dgate")
        else:
            dgate, d_dgate = param(dgate, "dgate")
    if w_post is not None:
        dw_post, d_post = param(dw_post, "dw_post")
    if w_pre is not None:
        dw_pre, d_pre = param(dw_pre, "dw_pre")
    g = E.ecc_norm_grad_t(d_dh, ld_dh, d_dxo, ld_dxo, d_dx, ld_dx, d_df, ld_df, d_dgate, ld_dgate,
                          d_post, d_pre, _type(dtype, "the gradients"), 1 if accumulate else 0,
                          D if apart else stride)
    _one_gpu(x, (f, dh, dx_out, w_post, w_pre, gate, dx, df, dgate, dw_post, dw_pre),
             "x f dh dx_out w_post w_pre gate dx df dgate dw_post dw_pre")
    size = E.ecc_norm_work_size(a)
    # (a refused description has no size: the call says what is wrong)
    work = _work(max(size, 16), x) if work is None else _given_work(work, size, x)
    _launch(x, E.ecc_norm_grad, a, g, work)
    with torch.no_grad():
        for t, dense in copies:
            t.copy_(dense)
    return {"dx": dx, "df": df, "dgate": dgate, "dw_post": dw_post, "dw_pre": dw_pre}


# ----------------------------------------------------------------------------
# distillation
# ----------------------------------------------------------------------------

def distill(z, top, idx, tau=1.0, kd_weight=1.0, ce_weight=0.0, labels=None, weight=None,
            loss=None, grad=True, work=None):
    """(loss, gradient) of student logits z (..., V) against a teacher's top
    logits top (..., K) of the entries idx (..., K, int32; outside [0, V):
    absent): per position
    weight (kd_weight tau^2 KL + ce_weight * cross entropy of labels), and its
    gradient in z.  labels: int32, outside [0, V) for none; weight: fp32.
    grad: True (a new tensor), a tensor to write (z itself for in place), or
    None (loss only)."""
    t = _type(z, "z")
    N, ld_z = _rows(z, "z")
    V, shape = z.shape[-1], z.shape[:-1]
    if top.dim() < 1 or top.shape != idx.shape or top.shape[:-1] != shape:
        raise ValueError("top and idx must have K entries for every row of z, not shapes %s and "
                         "%s" % (tuple(top.shape), tuple(idx.shape)))
    if idx.dtype != torch.int32:
        raise TypeError("idx must be int32, not %s" % idx.dtype)
    for v, dtype, what in ((labels, torch.int32, "labels"), (weight, torch.float32, "weight")):
        if v is not None and (v.shape != shape or v.dtype != dtype):
            raise ValueError("%s must be %s of shape %s, not %s of %s" %
                             (what, dtype, tuple(shape), tuple(v.shape), v.dtype))
    a = E.ecc_distill_t(N, V, top.shape[-1], t, _type(top, "top"), 0, z.data_ptr(), ld_z,
                        _contiguous(top, "top").data_ptr(), _contiguous(idx, "idx").data_ptr(),
                        None if labels is None else _contiguous(labels, "labels").data_ptr(),
                        None if weight is None else _contiguous(weight, "weight").data_ptr(),
                        tau, kd_weight, ce_weight)
    loss = _out(loss, shape, torch.float64 if t == E.ECC_F64 else torch.float32, z, "loss")
    _contiguous(loss, "loss")
    ld_dz = 0
    if grad is True:
        grad = z.new_empty(z.shape)
    if grad is not None:
        _out(grad, z.shape, z.dtype, z, "grad")
        _, ld_dz = _rows(grad, "grad")
    _one_gpu(z, (top, idx, labels, weight, loss, grad), "z top idx labels weight loss grad")
    size = E.ecc_distill_work_size(a)
    # (a refused description has no size: the call says what is wrong)
    work = _work(max(size, 16), z) if work is None else _given_work(work, size, z)
    _launch(z, E.ecc_distill, a, loss, grad, ld_dz, work)
    return loss, grad
