#!/usr/bin/env python3
"""Data-parallel training of a small language model over the stale partial
allreduce, P workers on one GPU, each worker's gradient clipped by its own norm.

The model predicts the next token from the one before it: the token's embedding
x0, its norm h0, a gated feed-forward block f = (act(h0 Wg^T) h0 Wu^T) Wd^T, the
joint x1 = x0 + rms(f) w_post with its norm h1, and the logits h1 E^T of the same
token table E.  Each step
  - looks the tokens up, runs the joints, the block and one plain product
    (torch's);
  - takes loss and gradients from the hidden states, without the logits;
  - forms every worker's gradient of every parameter, the table's from both of
    its uses, and clips them into that worker's contribution to the allreduce
    (fp64; a worker whose gradient is not finite contributes zeros);
  - sums the contributions with ecc_allreduce_partial: a worker whose gradient
    does not arrive in time is stood in for by its last one, up to the slack;
  - steps the fp64 parameters, of which the kernels use an fp32 copy.

    python examples/train_lm.py [--steps N] [--slack S] [--arrive Q]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2203_17063_amd import capi as E     # noqa: E402
from paper_2203_17063_amd import lm            # noqa: E402
from paper_2203_17063_amd import runner        # noqa: E402


class Model:
    """Parameters in one fp64 vector, a contribution and a slot per worker."""

    def __init__(self, V, D, F, P, slack, seed, max_norm=1.0, act="silu", device="cuda"):
        self.V, self.D, self.P, self.max_norm, self.act = V, D, P, max_norm, act
        g = torch.Generator(device=device).manual_seed(seed)
        self.sizes = {"table": (V, D), "w_gate": (F, D), "w_up": (F, D), "w_down": (D, F),
                      "w0": (D,), "w_post": (D,), "w1": (D,)}
        self.m = sum(math.prod(s) for s in self.sizes.values())
        self.W = torch.empty(self.m, dtype=torch.float64, device=device)
        for p in self.views(self.W).values():
            if p.dim() == 2:
                p.normal_(0.0, 1.0 / math.sqrt(p.shape[1]), generator=g)
            else:
                p.fill_(1.0)
        self.contrib = torch.zeros((P, self.m), dtype=torch.float64, device=device)
        self.slots = torch.zeros_like(self.contrib)
        self.G = torch.empty_like(self.W)
        self.d_fresh = runner.ptr_array(list(self.contrib), device)
        self.d_slots = runner.ptr_array(list(self.slots), device)
        self.plan = runner.Plan(P, None, None, slack)
        self.scale = math.sqrt(D)

    def views(self, flat):
        """The parameters in a vector of them, or in P vectors as (P, ...)."""
        out, at = {}, 0
        for name, shape in self.sizes.items():
            n = math.prod(shape)
            out[name] = flat[..., at:at + n].unflatten(-1, shape)
            at += n
        return out

    def gradients(self, ids, labels):
        """The loss of each position and every worker's gradients, from its
        share of the sequences ids (B, T)."""
        P, V = self.P, self.V
        B, T = ids.shape
        if B % P:
            raise ValueError("%d sequences cannot be shared equally by %d workers" % (B, P))
        w = self.views(self.W.float())
        weight = torch.full(ids.shape, 1.0 / (B // P * T), device=ids.device)
        # forward: rows are positions, worker after worker
        x0 = lm.embed_lookup(w["table"], ids, scale=self.scale)
        _, h0 = lm.norm_forward(x0, w_pre=w["w0"])
        y = lm.gated_ffn(h0, w["w_gate"], w["w_up"], act=self.act)
        f = y @ w["w_down"].t()
        joint = dict(w_post=w["w_post"], w_pre=w["w1"])
        x1, h1 = lm.norm_forward(x0, f, **joint)
        loss, dh1, dtable = lm.cross_entropy(h1, w["table"], labels, weight, P=P)
        # backward
        g1 = lm.norm_grad(x1, f, dh1, None, P=P, **joint)
        df, rows = g1["df"].view(P, -1, self.D), y.view(P, -1, y.shape[-1])
        dw_down = torch.stack([df[p].t() @ rows[p] for p in range(P)])
        ffn = lm.gated_ffn_grad(h0, w["w_gate"], w["w_up"], g1["df"] @ w["w_down"], act=self.act,
                                P=P)
        g0 = lm.norm_grad(x0, None, ffn["dx"], g1["dx"], w_pre=w["w0"], P=P)
        index = lm.embed_index(ids, V, P=P)
        lm.embed_grad(index, g0["dx"], scale=self.scale, grad=dtable, accumulate=True)
        return loss, {"table": dtable, "w_gate": ffn["dw_gate"], "w_up": ffn["dw_up"],
                      "w_down": dw_down, "w0": g0["dw_pre"], "w_post": g1["dw_post"],
                      "w1": g1["dw_pre"]}

    def contribute(self, grads):
        """The gradients, clipped, into the contributions; their norms before."""
        places = self.views(self.contrib)
        return lm.clip_grads([grads[name] for name in places], self.max_norm, P=self.P,
                             out=list(places.values()), nonfinite="zero")

    def step(self, arrived, eta):
        """The (possibly stale) sum of the contributions, and a step along it."""
        E.ecc_allreduce_partial(self.plan.handle, self.m, self.d_fresh, self.d_slots, self.G,
                                arrived)
        self.W.add_(self.G, alpha=-eta / self.P)

    def close(self):
        self.plan.close()


BATCH = 64


def train(steps=100, P=8, slack=2, arrive=0.8, V=97, D=96, F=160, batch=BATCH, length=33, eta=0.5,
          seed=1):
    """The mean loss of every step, and the norms of the last one."""
    device = "cuda"
    model = Model(V, D, F, P, slack, seed, device=device)
    g = torch.Generator(device=device).manual_seed(seed + 1)
    # text: every token is followed by one of a few
    chance = torch.softmax(3.0 * torch.randn((V, V), generator=g, device=device), -1)
    losses, norms = [], None
    for _ in range(steps):
        ids = torch.randint(0, V, (batch, length), generator=g, device=device)
        labels = torch.multinomial(chance[ids.view(-1)], 1, generator=g)
        arrived = (torch.rand(P, generator=g, device=device) < arrive).to(torch.uint8)
        loss, grads = model.gradients(ids, labels.view(batch, length).to(torch.int32))
        norms = model.contribute(grads)
        model.step(arrived, eta)
        losses.append(loss.sum() / P)
    losses = torch.stack(losses).cpu().tolist()
    forced = model.plan.stats()[1]
    model.close()
    return losses, norms.cpu().tolist(), forced


def main():
    ap = argparse.ArgumentParser(description=__doc__,
                                 formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--slack", type=int, default=2)
    ap.add_argument("--arrive", type=float, default=0.8)
    a = ap.parse_args()
    if a.workers < 1 or BATCH % a.workers:
        ap.error("--workers must divide the %d sequences of a step" % BATCH)
    losses, norms, forced = train(a.steps, a.workers, a.slack, a.arrive)
    for t in range(0, a.steps, max(1, a.steps // 10)):
        print("step %4d  loss %.4f" % (t, losses[t]))
    print("last       loss %.4f  (%d gradients waited for, norms %.2f to %.2f)" %
          (losses[-1], forced, min(norms), max(norms)))


if __name__ == "__main__":
    main()
