"""The bounds of product_pieces.py see every product of pieces: without any one
of the six, results are outside of them.  No GPU."""
import pytest

torch = pytest.importorskip("torch")

import product_pieces as pp                               # noqa: E402

FFN = [(1, 40, 300, 49), (1, 130, 71, 90), (2, 100, 131, 70)]
CE = [(40, 300, 130), (130, 70, 90)]


@pytest.mark.parametrize("P,n,D,F", FFN)
def test_ffn(P, n, D, F):
    c = pp.ffn_case(P, n, D, F)
    assert pp.ffn_check(c, pp.ffn_emulate(c)) == []
    for stage in ("y", "dx", "dw_gate", "dw_up"):
        for lost in pp.SIX:
            which = tuple(p for p in pp.SIX if p != lost)
            bad = pp.ffn_check(c, pp.ffn_emulate(c, {stage: which}))
            assert [k for k, _ in bad] == [stage] and bad[0][1] > 2, (stage, lost, bad)


@pytest.mark.parametrize("N,D,V", CE)
def test_cross_entropy(N, D, V):
    for case, emulate, check in (
            (pp.ce_loss_case(N, D, V), pp.ce_loss_emulate, pp.ce_loss_check),
            (pp.ce_dh_case(N, D, V), pp.ce_dh_emulate, pp.ce_dh_check),
            (pp.ce_de_case(8, N, D, V), pp.ce_de_emulate, pp.ce_de_check),
            (pp.ce_de_case(3, N, D, V), pp.ce_de_emulate, pp.ce_de_check)):
        assert check(case, emulate(case)) == []
        for lost in pp.SIX:
            bad = check(case, emulate(case, tuple(p for p in pp.SIX if p != lost)))
            assert bad and bad[0][1] > 2, (emulate, lost, bad)


def test_bf16_rows():
    """fp32 gradients of bf16 rows: three pieces of the gradients' terms beside one
    of the rows."""
    f = pp.ffn_case(2, 100, 131, 70, torch.bfloat16)
    c = pp.ce_de_case(8, 40, 300, 130, torch.bfloat16)
    ours = ("dw_gate", "dw_up")

    def ffn(which):
        got = pp.ffn_emulate(f, {k: which for k in ours})
        return pp.ffn_check(f, {k: got[k] for k in ours})
    assert ffn(pp.SIX) == [] and pp.ce_de_check(c, pp.ce_de_emulate(c)) == []
    for lost in ((2, 0), (1, 0), (0, 0)):
        which = tuple(p for p in pp.SIX if p != lost)
        assert len(ffn(which)) == 2 and pp.ce_de_check(c, pp.ce_de_emulate(c, which)) != []
