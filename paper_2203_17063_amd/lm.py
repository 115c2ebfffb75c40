"""Operators of language models over the C ABI: shapes, types and strides are
read from torch tensors and checked, outputs and work buffers allocated, and
libecc called on the current stream.  No arithmetic runs here.

The calls are not recorded for torch's differentiation: results of inputs that
require gradients do not, and the gradients are the calls named *_grad (and
further results of distill and cross_entropy).

Rows (tokens, positions) may come with any number of leading dimensions as
long as the last one is contiguous and the others collapse to rows of one
stride.  Operands, outputs and work buffers of a call lie on one GPU, which
need not be the current one.  Sums over rows and tokens are held in fp32, or
fp64 where an operand or the result is fp64; a row's own sums (norms, softmax
statistics) in fp32, or fp64 for rows of fp64; norms of whole gradients in fp64.
cross_entropy and gated_ffn are products of fp32 or bf16 operands, not fp64;
fp32 ones must be finite (an infinite element makes its sums NaN).
"""
from __future__ import annotations

import struct

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


# ----------------------------------------------------------------------------
# cross entropy from hidden states
# ----------------------------------------------------------------------------

def _product_type(t, what):
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("%s must be float32 or bfloat16, not %s" % (what, t.dtype))
    return _TYPES[t.dtype]


def cross_entropy(h, table, labels, weight=None, scale=1.0, P=1, grad=True, dtype=None, loss=None,
                  dh=None, dtable=None, accumulate=False, work=None):
    """(loss, dh, dtable) of the logits scale * h table^T, which exist for a piece
    of rows at a time (with their gradients 5 GiB of the work buffer at most, or
    256 rows of a vocabulary for which those are more): per row of h (..., D)
    weight (log sum exp of its logits - the logit of its label), and the gradients
    of the losses' sum in h and, per worker (P, V, D), in the table.

    labels: int32, outside [0, V) for none; weight: fp32.  grad: None for the
    loss only.  dtype: of dtable, float32 or the table's (which it is by
    default); dtable: written, or with accumulate added to; its rows and
    workers may be strided."""
    if table.dim() != 2:
        raise ValueError("table must be a matrix")
    V, D = table.shape
    t = _product_type(h, "h")
    if table.dtype != h.dtype:
        raise TypeError("table must be %s like h, not %s" % (h.dtype, table.dtype))
    N, ld_h = _rows(h, "h", D)
    _, ld_table = _rows(table, "table")
    shape = h.shape[:-1]
    for v, kind, what in ((labels, torch.int32, "labels"), (weight, torch.float32, "weight")):
        if v is None and what == "weight":
            continue
        if v.shape != shape or v.dtype != kind:
            raise ValueError("%s must be %s of shape %s, not %s of %s" %
                             (what, kind, tuple(shape), tuple(v.shape), v.dtype))
        _contiguous(v, what)
    if P < 1 or N % P:
        raise ValueError("%d rows cannot be shared equally by %d workers" % (N, P))
    if not grad and (dh is not None or dtable is not None or accumulate):
        raise ValueError("gradients given without grad")
    if dtable is not None:
        if tuple(dtable.shape) != (P, V, D):
            raise ValueError("dtable must have shape %s, not %s" % ((P, V, D), tuple(dtable.shape)))
        if D > 1 and dtable.stride(2) != 1:
            raise ValueError("dtable must be contiguous in its last dimension")
        dtype = dtable.dtype
    elif accumulate:
        raise ValueError("accumulate needs dtable")
    dtype = dtype or table.dtype
    if dtype not in (torch.float32, table.dtype):
        raise TypeError("dtable must be float32 or %s, not %s" % (table.dtype, dtype))
    loss = _out(loss, shape, torch.float32, h, "loss")
    _contiguous(loss, "loss")
    ld_dh = ld_dt = stride = 0
    if grad:
        dh = _out(dh, h.shape, h.dtype, h, "dh")
        _, ld_dh = _rows(dh, "dh")
        if dtable is None:
            dtable = table.new_empty((P, V, D), dtype=dtype)
        ld_dt = dtable.stride(1) if V > 1 else D
        stride = dtable.stride(0) if P > 1 else V * D
    _one_gpu(h, (table, labels, weight, loss, dh, dtable), "h table labels weight loss dh dtable")
    a = E.ecc_cross_entropy_t(N // P, V, D, P, t, _TYPES[dtype], 0, h.data_ptr(), ld_h,
                              table.data_ptr(), ld_table, labels.data_ptr(),
                              None if weight is None else weight.data_ptr(), scale)
    size = E.ecc_cross_entropy_work_size(a, 1 if grad else 0)
    # (a refused description has no size: the call says what is wrong)
    work = _work(max(size, 16), h) if work is None else _given_work(work, size, h)
    _launch(h, E.ecc_cross_entropy, a, loss, dh, ld_dh, dtable, ld_dt, stride,
            1 if accumulate else 0, work)
    return loss, dh, dtable


# ----------------------------------------------------------------------------
# the gated feed-forward block
# ----------------------------------------------------------------------------

_ACTS = {"silu": E.ECC_ACT_SILU, "gelu": E.ECC_ACT_GELU}


def _ffn(x, w_gate, w_up, act, P, dtype):
    """The ecc_ffn_t of tensors; rows and inner width."""
    if w_gate.dim() != 2 or w_gate.shape != w_up.shape:
        raise ValueError("w_gate and w_up must be matrices of one shape, not %s and %s" %
                         (tuple(w_gate.shape), tuple(w_up.shape)))
    F, D = w_gate.shape
    t = _product_type(x, "x")
    if w_gate.dtype != x.dtype or w_up.dtype != x.dtype:
        raise TypeError("the weights must be %s like x, not %s and %s" %
                        (x.dtype, w_gate.dtype, w_up.dtype))
    if act not in _ACTS:
        raise ValueError("act must be one of %s, not %r" % (", ".join(_ACTS), act))
    if dtype not in (torch.float32, x.dtype):
        raise TypeError("the weights' gradients must be float32 or %s, not %s" % (x.dtype, dtype))
    N, ld_x = _rows(x, "x", D)
    if P < 1 or N % P:
        raise ValueError("%d rows cannot be shared equally by %d workers" % (N, P))
    a = E.ecc_ffn_t(N // P, D, F, P, t, _TYPES[dtype], _ACTS[act], x.data_ptr(), ld_x,
                    w_gate.data_ptr(), _rows(w_gate, "w_gate")[1], w_up.data_ptr(),
                    _rows(w_up, "w_up")[1])
    return a, N, F


def gated_ffn(x, w_gate, w_up, act="silu", out=None, work=None):
    """act(x w_gate^T) * (x w_up^T), of shape (..., F), for weights (F, D).
    act: "silu" or "gelu" (by erf, within 7.5e-8 |x w_gate^T|)."""
    a, _, F = _ffn(x, w_gate, w_up, act, 1, x.dtype)
    out = _out(out, x.shape[:-1] + (F,), x.dtype, x, "out")
    _, ld = _rows(out, "out")
    _one_gpu(x, (w_gate, w_up, out), "x w_gate w_up out")
    size = E.ecc_ffn_work_size(a, 0)
    # (a refused description has no size: the call says what is wrong)
    work = _work(max(size, 16), x) if work is None else _given_work(work, size, x)
    _launch(x, E.ecc_ffn_forward, a, out, ld, work)
    return out


def gated_ffn_grad(x, w_gate, w_up, dy, act="silu", P=1, dtype=None, dx=None, dw_gate=None,
                   dw_up=None, accumulate=False, work=None):
    """The gradients of gated_ffn for a given dy: a dict of dx, and dw_gate and
    dw_up per worker, (P, F, D) of dtype (float32, or the weights' type, which
    it is by default).  Given ones of the weights may be views of contributions
    whose workers lie one common stride apart, and accumulate adds to them."""
    given = [w for w in (dw_gate, dw_up) if w is not None]
    if len(given) == 1 or (accumulate and not given):
        raise ValueError("the weights' gradients are given together" if given else
                         "accumulate needs dw_gate and dw_up")
    dtype = given[0].dtype if given else dtype or w_gate.dtype
    a, N, F = _ffn(x, w_gate, w_up, act, P, dtype)
    D = w_gate.shape[1]
    rows, ld_dy = _rows(dy, "dy", F)
    if rows != N or dy.dtype != x.dtype:
        raise ValueError("dy must have %d rows of %s, not %s of %s" %
                         (N, x.dtype, tuple(dy.shape), dy.dtype))
    dx = _out(dx, x.shape, x.dtype, x, "dx")
    _, ld_dx = _rows(dx, "dx")
    if not given:
        dw_gate, dw_up = (x.new_empty((P, F, D), dtype=dtype) for _ in range(2))
    stride = dw_gate.stride(0) if P > 1 else F * D
    for w in (dw_gate, dw_up):
        if tuple(w.shape) != (P, F, D) or w.dtype != dtype or not w[0].is_contiguous() or \
                (P > 1 and w.stride(0) != stride):
            raise ValueError("dw_gate and dw_up must be dense matrices of %s per worker, of shape "
                             "%s, one stride for both" % (dtype, (P, F, D)))
    _one_gpu(x, (w_gate, w_up, dy, dx, dw_gate, dw_up), "x w_gate w_up dy dx dw_gate dw_up")
    size = E.ecc_ffn_work_size(a, 1)
    # (a refused description has no size: the call says what is wrong)
    work = _work(max(size, 16), x) if work is None else _given_work(work, size, x)
    _launch(x, E.ecc_ffn_grad, a, dy, ld_dy, dx, ld_dx, dw_gate, dw_up, stride,
            1 if accumulate else 0, work)
    return {"dx": dx, "dw_gate": dw_gate, "dw_up": dw_up}


# ----------------------------------------------------------------------------
# norms and clipping of gradients
# ----------------------------------------------------------------------------

def _worker_parts(t, P, what):
    """(elements per worker, elements from one worker to the next)."""
    if P is None:
        return _contiguous(t, what).numel(), 0
    if t.dim() < 1 or t.shape[0] != P:
        raise ValueError("%s must have %d workers in its first dimension, not shape %s" %
                         (what, P, tuple(t.shape)))
    n = t.numel() // P
    if t.is_contiguous():
        return n, n
    if not t[0].is_contiguous():
        raise ValueError("%s must be contiguous for each worker" % what)
    return n, t.stride(0)


# An ecc_tensor_t: two addresses, three sizes, two types.
_TENSOR = struct.Struct("=QQqqqii")


def _tensors(grads, out, P):
    """The array of ecc_tensor_t, their number, and the first tensor."""
    grads = list(grads)
    if not grads:
        raise ValueError("there are no gradients")
    if P is not None and P < 1:
        raise ValueError("P must be >= 1")
    count = len(grads)
    outs = (None,) * count if out is None else list(out)
    if len(outs) != count:
        raise ValueError("%d outputs for %d gradients" % (len(outs), count))
    device = grads[0].get_device()
    if device < 0:
        raise ValueError("grads must be on the GPU")
    data, at, size = bytearray(count * _TENSOR.size), 0, _TENSOR.size
    pack, types = _TENSOR.pack_into, _TYPES
    for g, o in zip(grads, outs):
        if g.get_device() != device:
            raise ValueError("grads must be on one GPU")
        shape = g.shape
        if P is None:
            n, stride = _contiguous(g, "a gradient").numel(), 0
        elif len(shape) and shape[0] == P and g.is_contiguous():
            n = stride = g.numel() // P
        else:
            n, stride = _worker_parts(g, P, "a gradient")
        kind = types.get(g.dtype)
        if kind is None:
            _type(g, "a gradient")
        if o is None:
            pack(data, at, g.data_ptr(), 0, n, stride, 0, kind, 0)
        else:
            if o.shape != shape:
                raise ValueError("an output must have its gradient's shape %s, not %s" %
                                 (tuple(shape), tuple(o.shape)))
            if o.get_device() != device:
                raise ValueError("grads and out must be on one GPU")
            out_kind = types.get(o.dtype)
            if out_kind is None:
                _type(o, "an output")
            pack(data, at, g.data_ptr(), o.data_ptr(), n, stride,
                 n if o.is_contiguous() else _worker_parts(o, P, "an output")[1], kind, out_kind)
        at += size
    return (E.ecc_tensor_t * count).from_buffer(data), grads[0]


def _norms(norms, P, like):
    norms = _out(norms, (1 if P is None else P,), torch.float64, like, "norms")
    _contiguous(norms, "norms")
    _one_gpu(like, (norms,), "grads norms")
    return norms


def grad_norm(grads, P=None, norms=None, work=None):
    """The global norm over the tensors `grads`, float64 of shape (1,), or with
    P given, tensors of shape (P, ...), each worker's, of shape (P,)."""
    a, like = _tensors(grads, None, P)
    norms = _norms(norms, P, like)
    size = E.ecc_grad_norm_work_size(P or 1, len(a), a)
    # (refused tensors have no size: the call says what is wrong)
    work = _work(max(size, 16), like) if work is None else _given_work(work, size, like)
    _launch(like, E.ecc_grad_norm, P or 1, len(a), a, norms, work)
    return norms


_NONFINITE = {"keep": E.ECC_CLIP_KEEP, "zero": E.ECC_CLIP_ZERO}


def clip_grads(grads, max_norm, P=None, out=None, nonfinite="keep", norms=None, work=None):
    """Scales gradients to at most max_norm, each worker's by its own norm, and
    returns the norms before that (see grad_norm).

    out: tensors of the gradients' shapes and any type to write instead (e.g.
    the parameters' places in the workers' contributions); None in a place, or
    for all: in place.  nonfinite: "keep" leaves the gradients of a worker whose
    norm is infinite or NaN as they are, "zero" makes them zeros."""
    if nonfinite not in _NONFINITE:
        raise ValueError("nonfinite must be one of %s, not %r" %
                         (", ".join(_NONFINITE), nonfinite))
    a, like = _tensors(grads, out, P)
    norms = _norms(norms, P, like)
    size = E.ecc_grad_norm_work_size(P or 1, len(a), a)
    # (refused tensors have no size: the call says what is wrong)
    work = _work(max(size, 16), like) if work is None else _given_work(work, size, like)
    _launch(like, E.ecc_clip_grads, P or 1, len(a), a, max_norm, _NONFINITE[nonfinite], norms,
            work)
    return norms
