"""fp32 products through the library's calls, one to three terms at a time, so that
a lost piece of an operand shows (test_product_pieces.py: each of the six products
of pieces, left out, puts results outside of these bounds)."""
import pytest

torch = pytest.importorskip("torch")

import product_pieces as pp                               # noqa: E402
from gpu_common import announce                           # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


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


# Few rows straight from memory; small tiles; products split along k; large tiles,
# alone and split; workers.
FFN = [(1, 40, 300, 49), (1, 130, 71, 90), (2, 100, 131, 70), (1, 70, 4097, 100),
       (1, 2000, 701, 1500), (3, 700, 512, 1201), (1, 4000, 800, 2001), (8, 517, 1001, 2731),
       (1, 16400, 512, 67)]


def _ffn(c, dtype=None):
    x, dy, wg, wu = (c[k].cuda() for k in ("x", "dy", "wg", "wu"))
    got = _lm().gated_ffn_grad(x, wg, wu, dy, P=c["P"], dtype=dtype)
    return dict(got, y=_lm().gated_ffn(x, wg, wu))


@pytest.mark.parametrize("P,n,D,F", FFN)
def test_ffn(P, n, D, F):
    announce("pieces, ffn", P, n, D, F)
    c = pp.ffn_case(P, n, D, F)
    assert pp.ffn_check(c, _ffn(c)) == []


@pytest.mark.parametrize("P,n,D,F", FFN)
def test_ffn_of_bf16(P, n, D, F):
    """fp32 gradients of bf16 weights."""
    announce("pieces, ffn of bf16", P, n, D, F)
    c = pp.ffn_case(P, n, D, F, BF16)
    got = _ffn(c, F32)
    assert pp.ffn_check(c, {k: got[k] for k in ("dw_gate", "dw_up")}) == []


CE = [(1, 40, 300, 130), (1, 9, 65, 2500), (1, 64, 4100, 200), (4, 16, 70, 300), (1, 130, 70, 90),
      (1, 700, 250, 3001), (1, 130, 3001, 200), (2, 700, 1000, 4001), (1, 3000, 600, 4000),
      (3, 100, 64, 200)]


@pytest.mark.parametrize("P,n,D,V", CE)
def test_cross_entropy(P, n, D, V):
    announce("pieces, cross entropy", P, n, D, V)
    lm = _lm()

    def run(c, **kw):
        return lm.cross_entropy(c["h"].cuda(), c["table"].cuda(), c["y"].cuda(), **kw)
    c = pp.ce_loss_case(P * n, D, V)
    for grad in (True, None):
        assert pp.ce_loss_check(c, {"loss": run(c, P=P, grad=grad)[0]}) == []
    c = pp.ce_dh_case(P * n, D, V)
    assert pp.ce_dh_check(c, {"dh": run(c, P=P)[1]}) == []
    for dtype in (F32, BF16):
        c = pp.ce_de_case(P, n, D, V, dtype)
        assert pp.ce_de_check(c, {"dtable": run(c, P=P, dtype=F32)[2]}) == []
