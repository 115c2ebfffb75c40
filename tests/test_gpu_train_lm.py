"""A whole training step through the language-model operators: the example's
gradients and contributions against the same model in 64 bits with torch's own
differentiation, eager and in a replayed graph."""
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


def _batch(V, B, T, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, V, (B, T), generator=g, device="cuda")
    labels = torch.randint(-1, V, (B, T), generator=g, device="cuda")
    return ids, labels.to(torch.int32)


def _reference(model, ids, labels, p):
    """Worker p's loss and gradient by torch's differentiation on the CPU."""
    per = ids.shape[0] // model.P
    own = slice(p * per, (p + 1) * per)
    flat = model.W.cpu().float().double().requires_grad_(True)
    w = model.views(flat)
    i, y = ids[own].cpu(), labels[own].cpu().long()

    def rms(v):
        return v / (v.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()

    x0 = w["table"][i] * model.scale
    h0 = rms(x0) * w["w0"]
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[model.act]
    f = (act(h0 @ w["w_gate"].t()) * (h0 @ w["w_up"].t())) @ w["w_down"].t()
    h1 = rms(x0 + rms(f) * w["w_post"]) * w["w1"]
    logq = torch.log_softmax(h1 @ w["table"].t(), -1)
    nll = -logq.gather(-1, y.clamp(min=0)[..., None])[..., 0]
    loss = torch.where(y >= 0, nll, 0.0) / i.numel()
    g, = torch.autograd.grad(loss.sum(), flat)
    return loss.detach(), g


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_step_against_differentiation(act):
    """fp32 activations through two norms and four products of 96 to 331 terms:
    relative errors of some 1e-6 in the sums; 1e-4 of the largest element leaves
    room for the cancellation in a gradient of a hundred tokens."""
    import train_lm as X
    announce("trained model, one step", act)
    V, D, F, P = 331, 96, 130, 4
    model = X.Model(V, D, F, P, 0, 4, max_norm=0.05, act=act)
    ids, labels = _batch(V, 8, 33, 5)
    loss, grads = model.gradients(ids, labels)
    norms = model.contribute(grads)
    total = torch.zeros(model.m, dtype=torch.float64)
    for p in range(P):
        want_l, want_g = _reference(model, ids, labels, p)
        got_l = loss[2 * p:2 * p + 2].cpu().double()
        assert (got_l - want_l).abs().max() <= 1e-4 * want_l.abs().max()
        norm = float(want_g.norm())
        assert norm > model.max_norm and abs(float(norms[p]) - norm) <= 1e-4 * norm
        got = model.views(model.contrib[p].cpu())
        clipped = want_g * (model.max_norm / norm)
        for name, want in model.views(clipped).items():
            err = (got[name] - want).abs().max()
            assert err <= 1e-4 * want.abs().max(), (p, name, float(err))
        total += clipped
    before = model.W.clone()
    model.step(torch.ones(P, dtype=torch.uint8, device="cuda"), 0.25)
    moved = ((before - model.W) / 0.25 * P).cpu()
    assert (moved - total).abs().max() <= 1e-4 * total.abs().max()
    model.close()


def test_step_in_a_graph():
    """Gradients and contributions of a captured step are those of the eager
    one, replay after replay."""
    import train_lm as X
    announce("trained model, captured")
    V, P = 211, 2
    model = X.Model(V, 64, 100, P, 0, 6, max_norm=0.1)
    ids, labels = _batch(V, 4, 40, 7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        model.contribute(model.gradients(ids, labels)[1])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, grads = model.gradients(ids, labels)
        norms = model.contribute(grads)
    for k in range(3):
        ids2, labels2 = _batch(V, 4, 40, 8 + k)
        ids.copy_(ids2)
        labels.copy_(labels2)
        graph.replay()
        torch.cuda.synchronize()
        got = [loss.clone(), norms.clone(), model.contrib.clone()]
        want_l, want_g = model.gradients(ids, labels)
        want = [want_l, model.contribute(want_g), model.contrib]
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    model.close()


def test_a_worker_that_is_lost():
    """A worker whose gradient is not finite contributes zeros, the others as
    ever."""
    import train_lm as X
    announce("trained model, a lost worker")
    model = X.Model(101, 32, 48, 3, 0, 9)
    ids, labels = _batch(101, 6, 20, 10)
    _, grads = model.gradients(ids, labels)
    model.contribute(grads)
    want = model.contrib.clone()
    grads["w_up"][1, 3, 5] = float("nan")
    norms = model.contribute(grads)
    assert torch.isnan(norms[1]) and (model.contrib[1] == 0).all()
    assert torch.equal(model.contrib[0], want[0]) and torch.equal(model.contrib[2], want[2])
    model.close()


@pytest.mark.parametrize("slack,arrive", [(0, 1.0), (2, 0.7)])
def test_training_runs(slack, arrive):
    """The same run gives the same losses, with fresh gradients and stale ones."""
    import train_lm as X
    announce("trained model, training", slack, arrive)
    losses, norms, forced = X.train(12, slack=slack, arrive=arrive)
    assert all(0 < v < 20 for v in losses) and all(0 < v < 1e3 for v in norms)
    assert forced == 0 or arrive < 1.0
    assert X.train(5, slack=slack, arrive=arrive)[0] == losses[:5]
