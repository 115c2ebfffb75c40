"""Sizes and refusals of the language-model operators that need no GPU: the
size calls, and argument errors found before anything is enqueued."""
import os
import sys

import pytest

from paper_2203_17063_amd import capi as E


def test_index_and_work_sizes():
    # keys, tokens and a flag per row; twice the first two beyond the LDS sort
    assert E.ecc_embed_index_size(1, 100, 50) >= 100 * 8 + 50
    assert E.ecc_embed_index_size(4, 20000, 50) >= 4 * 20000 * 16
    assert E.ecc_embed_index_size(1, 0, 50) >= 1
    for bad in ((0, 5, 5), (1, -1, 5), (1, 5, 0), (1, 1 << 31, 5), (1, 5, (1 << 31) - 1),
                (1 << 16, 1, 1 << 15), (3, 1 << 30, 5)):
        assert E.ecc_embed_index_size(*bad) == -1, bad
    # two pieces of a tile, in the accumulator's type
    f32 = E.ecc_embed_work_size(1, 1000, 64, E.ECC_BF16, E.ECC_F32)
    assert f32 >= 2 * 64 * 4 * (1000 // 64)
    assert E.ecc_embed_work_size(1, 1000, 64, E.ECC_BF16, E.ECC_F64) == 2 * f32
    for bad in ((0, 5, 5, 1, 1), (1, -1, 5, 1, 1), (1, 5, 0, 1, 1), (1, 5, (1 << 22) + 1, 1, 1),
                (1, 5, 5, 3, 1), (1, 5, 5, 1, 4), (3, 1 << 30, 5, 1, 1)):
        assert E.ecc_embed_work_size(*bad) == -1, bad


def _norm(**kw):
    d = dict(n=100, D=64, P=2, type=E.ECC_F32, w_type=E.ECC_F32, d_x=64, ld_x=64, d_f=64, ld_f=64,
             d_gate=None, ld_gate=0, gate_rows=0, d_w_post=None, d_w_pre=64, w_offset=0.0,
             res_scale=1.0, branch_scale=1.0, eps=1e-6)
    d.update(kw)
    return E.ecc_norm_t(**d)


def test_norm_work_size():
    assert E.ecc_norm_work_size(_norm()) >= 3 * 2 * 64 * 4
    assert E.ecc_norm_work_size(_norm(n=0)) >= 16
    assert E.ecc_norm_work_size(_norm(D=E.ECC_NORM_MAX_DIM, ld_x=1 << 15, ld_f=1 << 15)) > 0
    for bad in (dict(n=-1), dict(P=0), dict(D=0), dict(type=5), dict(eps=0.0), dict(ld_x=63),
                dict(D=E.ECC_NORM_MAX_DIM + 1, ld_x=1 << 15, ld_f=1 << 15),
                dict(type=E.ECC_F64, D=E.ECC_NORM_MAX_DIM // 2 + 1, ld_x=1 << 15, ld_f=1 << 15),
                dict(d_gate=64, gate_rows=3, ld_gate=64)):
        assert E.ecc_norm_work_size(_norm(**bad)) == -1, bad
        assert E.ecc_last_error() != ""


@pytest.mark.parametrize("N,V,split", [(1, 100, False), (1, 128000, True), (600, 128000, False),
                                       (0, 100, False)])
def test_distill_work_size(N, V, split):
    a = E.ecc_distill_t(N, V, 16, E.ECC_F32, E.ECC_F32, 0, 64, V, 64, 64, None, None, 1.0, 1.0,
                        0.0)
    size = E.ecc_distill_work_size(a)
    assert (size > 16) == split
    if split:
        assert size >= N * (3 * 2 + 17) * 4


def test_refused_without_a_device():
    lib = E.lib()
    assert lib.ecc_embed_lookup(-1, 1, 1, 0, None, E.ECC_I32, None, 1, 1, 1.0, None, 1, 1,
                                None) == E.ECC_ERR_ARG
    assert lib.ecc_embed_lookup(4, 8, 8, 0, None, E.ECC_I32, 64, 1, 8, 1.0, 64, 1, 8,
                                None) == E.ECC_ERR_ARG
    assert lib.ecc_embed_index(1, 1 << 31, 5, 0, 64, E.ECC_I32, 64, None) == E.ECC_ERR_RANGE
    assert lib.ecc_embed_grad(1, 4, 8, 8, 64, 64, 1, 7, 1.0, 64, 1, 8, 64, 0, 64,
                              None) == E.ECC_ERR_ARG
    assert lib.ecc_norm_forward(_norm(eps=-1.0), 64, 64, 64, 64, None) == E.ECC_ERR_ARG
    assert lib.ecc_norm_forward(None, 64, 64, 64, 64, None) == E.ECC_ERR_ARG
    assert lib.ecc_norm_grad(_norm(), None, 64, None) == E.ECC_ERR_ARG
    assert lib.ecc_distill(None, 64, 64, 8, 64, None) == E.ECC_ERR_ARG
    assert lib.ecc_distill_work_size(None) == -1
    # nothing to do is no error, with nothing to point to
    assert lib.ecc_embed_lookup(0, 8, 8, 0, None, E.ECC_I32, None, 1, 8, 1.0, None, 1, 8,
                                None) == E.ECC_OK


def test_example_shares_its_sequences():
    """A batch that the workers cannot share equally is refused: their
    gradients would be of different sequences in the different operators."""
    torch = pytest.importorskip("torch")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                    "examples"))
    import distill_lm
    student = object.__new__(distill_lm.Student)
    student.P, student.V, student.D = 3, 7, 4
    with pytest.raises(ValueError, match="64 sequences"):
        student.gradients(torch.zeros((64, 33), dtype=torch.int64), None, None, None, None, 1.0,
                          1.0, 0.0)
    for workers in ("3", "0", "-8", "65"):
        with pytest.raises(SystemExit):
            sys.argv, argv = ["distill_lm.py", "--workers", workers], sys.argv
            try:
                distill_lm.main()
            finally:
                sys.argv = argv


class _On:
    """What the device checks see of a tensor."""

    def __init__(self, device):
        self.device = device

    def get_device(self):
        return self.device


def test_operands_on_one_device(monkeypatch):
    lm = pytest.importorskip("paper_2203_17063_amd.lm")
    import contextlib
    lm._one_gpu(_On(1), (_On(1), None), "x f h")
    for other in (-1, 0, 2):
        with pytest.raises(ValueError, match="^gate must be on 1"):
            lm._one_gpu(_On(1), (_On(1), None, _On(other)), "x f h gate")
    with pytest.raises(ValueError, match="^x must be on the GPU"):
        lm._one_gpu(_On(-1), (_On(-1),), "x f")
    # a launch goes to the tensors' device and its stream
    now = [0]

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], d
        yield
        now[0] = before

    monkeypatch.setattr(lm.torch.cuda, "device", device)
    monkeypatch.setattr(lm, "_current_device", lambda: now[0])
    monkeypatch.setattr(lm, "_raw_stream", lambda d: 100 + d)
    seen = []
    for d in (0, 3):
        lm._launch(_On(d), lambda *args: seen.append((now[0],) + args), "a")
    assert seen == [(0, "a", 100), (3, "a", 103)] and now == [0]
