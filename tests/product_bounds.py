"""Errors of the library's products of matrices, for the tests' tolerances.

u = 2^-24.  A sum of n terms in fp32, added in any order by units that round
or cut off, is within 2 n u of the sum of its terms' magnitudes.  Products of
bf16 are exact in fp32.  fp32 operands are three bf16 pieces, the second at
most 2^-8 and the third at most 2^-16 of the element; of the nine products of
pieces those of 2^-24 or less are left out, 2^-23 + 2^-32 of the element's
product in all, and the other six make a sum of 6 n terms whose magnitudes add
up to at most (1 + 2^-6) of the products'."""
import torch

U = 2.0 ** -24
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
# half a step of a stored value
ULP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def product_error(n, dtype):
    """Of a product over n elements, relative to the sum of the magnitudes."""
    if dtype == BF16:
        return 2 * (n + 64) * U        # (rows are padded with zeros to 64)
    return (1 + 2.0 ** -6) * 12 * (n + 64) * U + 2.0 ** -23 + 2.0 ** -32


def product(a, b, dtype, ea=None, extra=0):
    """a @ b in 64 bits and the bound of its error, for an operand a off by up
    to ea; extra: other terms added in the same chain."""
    size = (a.abs() if ea is None else a.abs() + ea) @ b.abs()
    error = product_error(a.shape[-1] + extra, dtype) * size
    if ea is not None:
        error = error + ea @ b.abs()
    return a @ b, error


def within(got, want, error, what):
    """Stored values within half a step of something within `error` of `want`."""
    assert tuple(got.shape) == tuple(want.shape), what
    step = ULP[got.dtype]
    got, want, error = got.double().cpu(), want.cpu(), error.cpu()
    tol = error + step * (want.abs() + error) + 2.0 ** -120
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(((got - want).abs() / tol).max()))
