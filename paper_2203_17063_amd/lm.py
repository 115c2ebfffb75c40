"""Operators of language models over the C ABI: shapes, types and strides are
read from torch tensors and checked, outputs and work buffers allocated, and
libecc called on the current stream.  No arithmetic runs here.

Rows (tokens, positions) may come with any number of leading dimensions as
long as the last one is contiguous and the others collapse to rows of one
stride.  Sums are held in fp32, or fp64 where an operand or the result is
fp64.
"""
from __future__ import annotations

import torch

from . import capi as E

_TYPES = {torch.float64: E.ECC_F64, torch.float32: E.ECC_F32, torch.bfloat16: E.ECC_BF16}
_ID_TYPES = {torch.int32: E.ECC_I32, torch.int64: E.ECC_I64}


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _type(t, what):
    try:
        return _TYPES[t if isinstance(t, torch.dtype) else t.dtype]
    except KeyError:
        raise TypeError("%s must be float64, float32 or bfloat16, not %s" %
                        (what, t if isinstance(t, torch.dtype) else t.dtype)) from None


def _on_gpu(t, what):
    if not t.is_cuda:
        raise ValueError("%s must be on the GPU" % what)


def _rows(t, what, cols=None):
    """(rows, leading dimension) of a tensor seen as a matrix of its last
    dimension."""
    _on_gpu(t, what)
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
    _on_gpu(t, what)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % what)
    return t


def _out(t, shape, dtype, device, what):
    """The caller's output, checked, or a new one."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError("%s must be %s of shape %s, not %s of %s" %
                         (what, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    return t


def _work(size, device):
    if size < 0:
        raise E.EccError(E.ECC_ERR_RANGE, "the sizes are beyond what the library supports")
    return torch.empty(size, dtype=torch.uint8, device=device)


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
    out = _out(out, tuple(ids.shape) + (D,), dtype, ids.device, "out")
    _, ld_out = _rows(out, "out")
    E.ecc_embed_lookup(ids.numel(), V, D, row0, ids, id_type, table, tt, ld, scale, out, ot,
                       ld_out, _stream())
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
        index = EmbedIndex(P, n, V, _work(E.ecc_embed_index_size(P, n, V), ids.device))
    elif (index.P, index.n, index.V) != (P, n, V):
        raise ValueError("the index was made for other sizes")
    E.ecc_embed_index(P, n, V, row0, ids, id_type, index.data, _stream())
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
        grad = torch.empty((P, V, D), dtype=dtype, device=index.data.device)
    elif tuple(grad.shape) != (P, V, D):
        raise ValueError("grad must have shape %s, not %s" % ((P, V, D), tuple(grad.shape)))
    _on_gpu(grad, "grad")
    if D > 1 and grad.stride(2) != 1:
        raise ValueError("grad must be contiguous in its last dimension")
    yt, gt = _type(dy, "dy"), _type(grad, "grad")
    if work is None:
        work = _work(E.ecc_embed_work_size(P, n, D, yt, gt), grad.device)
    elif work.numel() * work.element_size() < E.ecc_embed_work_size(P, n, D, yt, gt):
        raise ValueError("the work buffer is too small")
    E.ecc_embed_grad(P, n, V, D, index.data, dy, yt, ld_dy, scale, grad, gt,
                     grad.stride(1) if V > 1 else D, grad.stride(0) if P > 1 else V * D,
                     1 if accumulate else 0, work, _stream())
    return grad
