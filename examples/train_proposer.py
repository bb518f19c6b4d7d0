"""Trains a small proposer for speculative decoding under a constraint, on one GPU.

    python examples/train_proposer.py

A "model" (here a fixed random one, whose next token depends on the last) decodes
under an automaton; a smaller proposer with one table for both its ends learns
to guess it: x = scale E[last] M, logits = x E^T, over the allowed tokens only.

  * The model's sampled tokens train it with the head loss (no logits kept); the
    embedding's gradient is added to the head's in place, the table being shared.
  * The model's top logits train it by distillation, loss and gradient in one
    pass that overwrites the logits.
  * ``spec_verify`` then counts how many of its proposals the model accepts.

The data (automaton, vocabulary, model) are synthetic.
"""
from __future__ import annotations

import math
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2403_06988_amd as dv  # noqa: E402
import workloads as W  # noqa: E402

BATCH, LENGTH, TOP, HIDDEN = 128, 16, 32, 128


class Model:
    """What the proposer learns from: logits from the last token alone."""

    def __init__(self, V, g, dev):
        self.table = torch.randn((V, 64), generator=g, device=dev).bfloat16()
        self.head = (torch.randn((V, 64), generator=g, device=dev) * (6.0 / 8.0)).bfloat16()

    def logits(self, last):
        return dv.embed(self.table, last) @ self.head.t()


class Proposer:
    def __init__(self, V, g, dev):
        self.scale = math.sqrt(HIDDEN)
        self.table = torch.randn((V, HIDDEN), generator=g, device=dev) / math.sqrt(HIDDEN)
        self.mix = torch.randn((HIDDEN, HIDDEN), generator=g, device=dev) / HIDDEN
        self.momentum = [torch.zeros_like(p) for p in (self.table, self.mix)]
        self.square = [torch.zeros_like(p) for p in (self.table, self.mix)]
        self.steps = 0

    def hidden(self, last):
        e = dv.embed(self.table, last, self.scale)
        return e, e @ self.mix

    def logits(self, last):
        return self.hidden(last)[1] @ self.table.t()

    def descend(self, grads, rate):
        """Adam on the table and the mixing matrix."""
        self.steps += 1
        for p, g, m, v in zip((self.table, self.mix), grads, self.momentum, self.square):
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.99).addcmul_(g, g, value=0.01)
            p.sub_(rate * (m / (1 - 0.9 ** self.steps)) / ((v / (1 - 0.99 ** self.steps)).sqrt() + 1e-8))

    def through_hidden(self, e, last, grad_x, grad_table):
        """The gradients below x, the embedding's added to the table's."""
        grad_mix = e.t() @ grad_x
        dv.embed_backward(grad_x @ self.mix.t(), last, self.table.shape[0], self.scale, grad_weight=grad_table,
                          accumulate=True)
        return grad_table, grad_mix

    def learn_tokens(self, last, targets, allow, states, rate):
        e, x = self.hidden(last)
        loss, lse = dv.head_loss(x, self.table, targets, allow, states)
        weights = torch.full_like(loss, 1.0 / loss.numel())
        grad_x, grad_table = dv.head_loss_backward(x, self.table, targets, lse, weights, allow, states)
        self.descend(self.through_hidden(e, last, grad_x, grad_table), rate)
        return loss.mean()

    def learn_logits(self, last, teacher_ids, teacher_logits, allow, states, rate):
        e, x = self.hidden(last)
        logits = x @ self.table.t()
        weights = torch.full((last.numel(),), 1.0 / last.numel(), device=last.device)
        loss, grad = dv.distill_loss_backward(logits, teacher_ids, teacher_logits, weights, allow=allow, states=states,
                                              grad=logits)
        self.descend(self.through_hidden(e, last, grad @ self.table, grad.t() @ x), rate)
        return loss.mean()


def rollout(model, ns, al, start, g, step):
    """LENGTH sampled steps of BATCH sequences: last tokens, states, next
    tokens and the model's top logits, one row a step."""
    dev = start.device
    V = ns.shape[1]
    last = torch.randint(0, V, (BATCH,), generator=g, device=dev, dtype=torch.int32)
    states, rows = start, []
    for k in range(LENGTH):
        logits = model.logits(last)
        token, nxt = dv.masked_sample(ns, al, states, logits, seed=7, offset=step * LENGTH + k)
        top = logits.float().topk(TOP, dim=1)
        rows.append((last, states, token, top.indices.int(), top.values))
        last, states = token, torch.where(nxt >= 0, nxt, start)  # a sequence that ended starts again
    return [torch.cat(c) for c in zip(*rows)]


def acceptance(model, proposer, ns, al, start, g, proposed=4):
    """Mean number of the proposer's greedy tokens that the model confirms."""
    dev = start.device
    first = torch.randint(0, ns.shape[1], (BATCH,), generator=g, device=dev, dtype=torch.int32)
    last, states, props, logits = first, start, [], [model.logits(first)]
    for _ in range(proposed):
        last, states = dv.masked_step(ns, al, states, proposer.logits(last))
        props.append(last)
        logits.append(model.logits(last))
    _, accepted, _ = dv.spec_verify(ns, al, start, torch.stack(props, 1).contiguous(), torch.stack(logits, 1).contiguous())
    return accepted.float().mean().item()


def main(steps=150, verbose=True):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(0)
    trans, _ = W.dfa(1)
    offsets, data = W.vocab(1)
    host = lambda a: torch.from_numpy(np.require(a, requirements=["C", "W"])).to(dev)  # noqa: E731
    ns, al = dv.align(host(trans), host(offsets), host(data))
    start = torch.zeros(BATCH, dtype=torch.int32, device=dev)
    model, proposer = Model(ns.shape[1], g, dev), Proposer(ns.shape[1], g, dev)
    report = dict(before=acceptance(model, proposer, ns, al, start, g), token_loss=[], distill_loss=[])
    for step in range(steps):
        last, states, targets, ids, top = rollout(model, ns, al, start, g, step)
        rate = 0.01 * (1 - step / steps)
        report["token_loss"].append(proposer.learn_tokens(last, targets, al, states, rate).item())
        report["distill_loss"].append(proposer.learn_logits(last, ids, top, al, states, rate).item())
        if verbose and step % 25 == 0:
            print(f"step {step:4d}  head loss {report['token_loss'][-1]:.3f}  distillation "
                  f"{report['distill_loss'][-1]:.3f}", flush=True)
    report["after"] = acceptance(model, proposer, ns, al, start, g)
    if verbose:
        print(f"proposals accepted of 4: {report['before']:.2f} before training, {report['after']:.2f} after", flush=True)
    return report


if __name__ == "__main__":
    main()
