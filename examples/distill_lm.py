#!/usr/bin/env python3
"""Data-parallel training of a small language model by distillation over the
stale partial allreduce, P workers on one GPU.

The student looks two tokens back: a token's embedding x0, the block f = (the
norm of the token before) B, the joint x1 = x0 + gate rms(f) w_post with its
norm h1, and the logits h1 E^T of the same token table E.  Its teacher gives
the top K logits of the next token after each pair of tokens.  Each step
  - looks the tokens up, runs both joints and the two plain products (torch's);
  - takes loss and logit gradient of all workers' positions in one call;
  - writes every worker's gradient of every parameter into that worker's
    contribution to the allreduce, the table's from both of its uses;
  - sums the contributions with ecc_allreduce_partial: a worker whose gradient
    does not arrive in time is stood in for by its last one, up to the slack;
  - steps the fp64 parameters, of which the kernels use an fp32 copy.

    python examples/distill_lm.py [--steps N] [--slack S] [--arrive Q]
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


class Teacher:
    """The top K logits of the next token after the tokens (before, now)."""

    def __init__(self, V, K, seed, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.now = 2.0 * torch.randn((V, V), generator=g, device=device)
        self.before = torch.randn((V, V), generator=g, device=device)
        self.K = K

    def __call__(self, before, now):
        top, idx = (self.now[now] + self.before[before]).topk(self.K, dim=-1)
        return top, idx.to(torch.int32)


class Student:
    """Parameters in one fp64 vector, a contribution and a slot per worker."""

    def __init__(self, V, D, P, slack, seed, device="cuda"):
        self.V, self.D, self.P = V, D, P
        g = torch.Generator(device=device).manual_seed(seed)
        self.sizes = {"table": (V, D), "block": (D, D), "w0": (D,), "w_post": (D,), "w1": (D,),
                      "gate": (D,)}
        self.m = sum(math.prod(s) for s in self.sizes.values())
        self.W = torch.empty(self.m, dtype=torch.float64, device=device)
        for name, p in self.views(self.W).items():
            if name in ("table", "block"):
                p.normal_(0.0, 1.0 / math.sqrt(D), generator=g)
            else:
                p.fill_(0.5 if name == "gate" else 1.0)
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

    def gradients(self, ids, top, idx, labels, weight, tau, kd_weight, ce_weight):
        """Every worker's gradient into its contribution, from its share of the
        sequences ids (B, T); the loss of each position."""
        P, V, D = self.P, self.V, self.D
        B, T = ids.shape
        if B % P:
            raise ValueError("%d sequences cannot be shared equally by %d workers" % (B, P))
        w = self.views(self.W.float())
        # forward: rows are positions, worker after worker
        x0 = lm.embed_lookup(w["table"], ids, scale=self.scale)
        _, h0 = lm.norm_forward(x0, w_pre=w["w0"])
        before = torch.zeros_like(h0)
        before[:, 1:] = h0[:, :-1]
        f = before @ w["block"]
        joint = dict(w_post=w["w_post"], w_pre=w["w1"], gate=w["gate"], gate_rows=0)
        x1, h1 = lm.norm_forward(x0, f, **joint)
        z = h1 @ w["table"].t()
        loss, dz = lm.distill(z, top, idx, tau, kd_weight, ce_weight, labels, weight, grad=z)
        # backward
        grad = self.views(self.contrib)
        per = B // P
        dh1 = dz @ w["table"]
        g1 = lm.norm_grad(x1, f, dh1, None, P=P, dw_post=grad["w_post"], dw_pre=grad["w1"],
                          dgate=grad["gate"], **joint)
        dh0 = torch.zeros_like(h0)
        dh0[:, :-1] = (g1["df"] @ w["block"].t())[:, 1:]
        g0 = lm.norm_grad(x0, None, dh0, g1["dx"], w_pre=w["w0"], P=P, dw_pre=grad["w0"])
        for p in range(P):
            own = slice(p * per, (p + 1) * per)
            grad["table"][p] = dz[own].reshape(-1, V).t() @ h1[own].reshape(-1, D)
            grad["block"][p] = before[own].reshape(-1, D).t() @ g1["df"][own].reshape(-1, D)
        index = lm.embed_index(ids, V, P=P)
        lm.embed_grad(index, g0["dx"], scale=self.scale, grad=grad["table"], accumulate=True)
        return loss

    def step(self, arrived, eta):
        """The (possibly stale) sum of the contributions, and a step along it."""
        E.ecc_allreduce_partial(self.plan.handle, self.m, self.d_fresh, self.d_slots, self.G,
                                arrived)
        self.W.add_(self.G, alpha=-eta)

    def close(self):
        self.plan.close()


BATCH = 64


def train(steps=100, P=8, slack=2, arrive=0.8, V=67, D=96, K=8, batch=BATCH, length=33, eta=4.0,
          tau=2.0, kd_weight=0.8, ce_weight=0.2, seed=1):
    """The mean loss of every step."""
    device = "cuda"
    teacher = Teacher(V, K, seed, device)
    student = Student(V, D, P, slack, seed + 1, device)
    g = torch.Generator(device=device).manual_seed(seed + 2)
    positions = batch * length
    losses = []
    for _ in range(steps):
        ids = torch.randint(0, V, (batch, length), generator=g, device=device)
        before = torch.cat([ids[:, :1], ids[:, :-1]], 1)
        top, idx = teacher(before, ids)
        # the hard label: a draw from the teacher's entries
        u = torch.rand(ids.shape, generator=g, device=device)
        at = (torch.softmax(top, -1).cumsum(-1) < u[..., None]).sum(-1).clamp_(max=K - 1)
        labels = idx.gather(-1, at[..., None])[..., 0]
        # a sequence's first position has no token before it
        weight = torch.full(ids.shape, 1.0 / positions, device=device)
        weight[:, 0] = 0.0
        arrived = (torch.rand(P, generator=g, device=device) < arrive).to(torch.uint8)
        loss = student.gradients(ids, top, idx, labels, weight, tau, kd_weight, ce_weight)
        student.step(arrived, eta)
        losses.append(loss.sum())
    losses = torch.stack(losses).cpu().tolist()
    clock, forced, _, _ = student.plan.stats()
    student.close()
    return losses, forced


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
    losses, forced = train(a.steps, a.workers, a.slack, a.arrive)
    for t in range(0, a.steps, max(1, a.steps // 10)):
        print("step %4d  loss %.4f" % (t, losses[t]))
    print("last       loss %.4f  (%d gradients waited for)" % (losses[-1], forced))


if __name__ == "__main__":
    main()
