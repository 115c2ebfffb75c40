"""The language-model operators together: the example's training step against
the same model in 64 bits with torch's own gradients, and its training."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

from gpu_common import announce                           # noqa: E402

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    yield
    torch.cuda.synchronize()


def _reference(student, ids, top, idx, labels, weight, tau, kd, ce, p):
    """Worker p's gradient by torch's differentiation in 64 bits on the CPU."""
    per = ids.shape[0] // student.P
    own = slice(p * per, (p + 1) * per)
    flat = student.W.cpu().float().double().requires_grad_(True)
    w = student.views(flat)
    i = ids[own].cpu()

    def rms(v):
        return v / (v.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()

    x0 = w["table"][i] * student.scale
    h0 = rms(x0) * w["w0"]
    before = torch.cat([torch.zeros_like(h0[:, :1]), h0[:, :-1]], 1)
    f = before @ w["block"]
    h1 = rms(x0 + w["gate"] * rms(f) * w["w_post"]) * w["w1"]
    z = h1 @ w["table"].t()
    t, k = top[own].cpu().double(), idx[own].cpu().long()
    logp = torch.log_softmax(t / tau, -1)
    logq = torch.log_softmax(z / tau, -1).gather(-1, k)
    loss = kd * tau ** 2 * (logp.exp() * (logp - logq)).sum(-1)
    y = labels[own].cpu().long()
    loss = loss - ce * torch.log_softmax(z, -1).gather(-1, y[..., None])[..., 0]
    loss = loss * weight[own].cpu().double()
    g, = torch.autograd.grad(loss.sum(), flat)
    return loss.detach(), g


def test_step_against_differentiation():
    """fp32 activations through two norms and three products of 96 and 331
    terms: relative errors of some 1e-6 in the sums; 1e-4 of the largest
    element leaves room for the cancellation in a gradient of a thousand
    tokens."""
    import distill_lm as X
    announce("distilled model, one step")
    V, D, P, K = 331, 96, 4, 16
    teacher, student = X.Teacher(V, K, 3), X.Student(V, D, P, 0, 4)
    g = torch.Generator(device="cuda").manual_seed(5)
    ids = torch.randint(0, V, (8, 33), generator=g, device="cuda")
    top, idx = teacher(torch.cat([ids[:, :1], ids[:, :-1]], 1), ids)
    labels = idx[..., 2].contiguous()
    weight = torch.full(ids.shape, 1.0 / ids.numel(), device="cuda")
    weight[:, 0] = 0.0
    loss = student.gradients(ids, top, idx, labels, weight, 2.0, 0.8, 0.2)
    total = torch.zeros(student.m, dtype=torch.float64)
    for p in range(P):
        want_l, want_g = _reference(student, ids, top, idx, labels, weight, 2.0, 0.8, 0.2, p)
        got_l = loss[2 * p:2 * p + 2].cpu().double()
        assert (got_l - want_l).abs().max() <= 1e-4 * want_l.abs().max()
        got = student.views(student.contrib[p].cpu())
        for name, want in student.views(want_g).items():
            err = (got[name] - want).abs().max()
            assert err <= 1e-4 * want.abs().max(), (p, name, float(err))
        total += want_g
    before = student.W.clone()
    student.step(torch.ones(P, dtype=torch.uint8, device="cuda"), 0.25)
    moved = ((before - student.W) / 0.25).cpu()
    assert (moved - total).abs().max() <= 1e-4 * total.abs().max()
    student.close()


@pytest.mark.parametrize("slack,arrive", [(0, 1.0), (2, 0.7)])
def test_training(slack, arrive):
    """The loss falls to less than half within 120 steps, with every gradient
    fresh and with stale ones; the same run gives the same losses."""
    import distill_lm as X
    announce("distilled model, training", slack, arrive)
    losses, forced = X.train(120, slack=slack, arrive=arrive)
    assert losses[-1] < 0.5 * losses[0]
    assert (forced == 0) == (arrive == 1.0)
    assert X.train(5, slack=slack, arrive=arrive)[0] == losses[:5]
