#!/usr/bin/env python
"""Decentralised policy fine-tuning of a small head on one GPU: n nodes, each with its own replica and its own data.

    python examples/policy_finetune.py [--nodes 8] [--rollouts 40] [--updates 4] [--dtype bf16]

Every node holds hidden states of its own, a layer norm and an output head on top of them (the replica: one row of the
stacked parameters x), draws a token for each state from its policy and is rewarded where the token is the one that a
planted rule names.  An update is the whole path of a training step:

    layer_norm -> head product -> policy_loss_grad -> head products -> layer_norm_grad -> gradient_clip -> decentlam_step

The layer norm's weights are read from column ranges of x; gradients of all tensors, fp32 and bf16 alike, are clipped by
their node's own norm and gathered into the rows of the stacked gradient g; the step mixes the replicas over a ring.
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2104_11981_b200 import binding as B  # noqa: E402


class Nodes:
    """n replicas of layer norm + head, their data, and the buffers of one update (all allocated once)."""

    def __init__(self, n=8, rows=64, width=256, vocab=32, dtype=torch.bfloat16, seed=0, device="cuda:0"):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.n, self.rows, self.width, self.vocab, self.dtype, self.gen = n, rows, width, vocab, dtype, gen
        normal = lambda shape, std: torch.empty(shape, device=device).normal_(0.0, std, generator=gen)  # noqa: E731
        self.hidden = normal((n, rows, width), 1.0).to(dtype)
        # the rule that names the right token, the same for all nodes: a random linear map, largest entry
        self.label = (self.hidden.float() @ normal((width, vocab), 1.0)).argmax(-1)
        # parameters: [weight | bias | head], one row a node, all replicas alike
        self.d = 2 * width + vocab * width
        self.x = torch.zeros((n, self.d), device=device)
        self.x[:, :width] = 1.0
        self.x[:, 2 * width:] = normal((1, vocab * width), 0.05)
        self.m, self.g = torch.zeros_like(self.x), torch.zeros_like(self.x)
        self.weight, self.bias = self.x[:, :width], self.x[:, width:2 * width]
        self.topology = B.topology_build(B.RING, n)
        self.iteration = 0
        acts = lambda *shape: torch.empty(shape, device=device, dtype=dtype)  # noqa: E731
        stat = lambda *shape: torch.empty(shape, device=device)  # noqa: E731
        self.y, self.dy, self.dhidden = acts(n, rows, width), acts(n, rows, width), acts(n, rows, width)
        self.logits, self.dhead = acts(n, rows, vocab), acts(n, vocab, width)
        self.mean, self.rstd, self.logp = stat(n, rows), stat(n, rows), stat(n, rows)
        self.dweight, self.dbias, self.loss, self.norms = stat(n, width), stat(n, width), stat(n), stat(n)
        work = max(B.layer_norm_grad_workspace_bytes(n, rows, width), B.policy_loss_workspace_bytes(n, rows, vocab))
        self.work = torch.empty(work, device=device, dtype=torch.uint8)
        self.list = B.gradients_build([[self.dweight[i], self.dbias[i], self.dhead[i]] for i in range(n)])
        assert self.list.columns == self.d
        self.ref = None  # reference log-probabilities of the tokens at hand

    def forward(self):
        """Logits of every node's hidden states under its replica."""
        B.layer_norm(self.hidden, self.weight, self.bias, 1e-5, self.y, self.mean, self.rstd)
        self.head = self.x[:, 2 * self.width:].reshape(self.n, self.vocab, self.width).to(self.dtype)
        torch.bmm(self.y, self.head.transpose(1, 2), out=self.logits)

    def score(self, tokens, keep, advantage=None, old=None, kl=0.0, grad=False):
        """Log-probabilities of tokens (and the loss and, in place of the logits, its gradient)."""
        zeros = torch.zeros_like(self.logp) if advantage is None or old is None else None
        B.policy_loss_grad(self.logits, tokens, keep, zeros if advantage is None else advantage, zeros if old is None else old,
                           self.ref if kl > 0.0 else None, 0.2, 0.28, kl, self.loss, self.logp,
                           self.logits if grad else None, self.work)
        return self.logp

    def gradients(self, tokens, keep, advantage, old, kl):
        """One forward and backward pass: fills loss, logp, dweight, dbias, dhead."""
        self.forward()
        self.score(tokens, keep, advantage, old, kl, grad=True)     # logits now hold dlogits
        torch.bmm(self.logits.transpose(1, 2), self.y, out=self.dhead)
        torch.bmm(self.logits, self.head, out=self.dy)
        B.layer_norm_grad(self.hidden, self.dy, self.weight, self.mean, self.rstd, self.dhidden, self.dweight, self.dbias,
                          self.work)

    def step(self, max_norm, beta, gamma):
        B.gradient_clip(self.list, max_norm, self.norms, self.g)
        B.decentlam_step(self.topology, self.iteration, self.x, self.m, self.g, beta, gamma)
        self.iteration += 1

    def rollout(self):
        """Tokens drawn from the current policy, which of them count, their advantages and log-probabilities."""
        self.forward()
        p = torch.softmax(self.logits.float(), -1).reshape(-1, self.vocab)
        tokens = torch.multinomial(p, 1, generator=self.gen).reshape(self.n, self.rows)
        keep = torch.full((self.n, self.rows), 1.0 / self.rows, device=tokens.device)
        reward = (tokens == self.label).float()
        advantage = (reward - reward.mean()) / reward.std().clamp(min=1e-3)
        old = self.score(tokens, keep).clone()
        return tokens, keep, advantage, old, reward.mean()

    def accuracy(self):
        """Probability of the right token, on average."""
        self.forward()
        keep = torch.ones((self.n, self.rows), device=self.x.device)
        return float(self.score(self.label, keep).exp().mean())

    def disagreement(self):
        return float((self.x - self.x.mean(0)).norm() / self.x.norm())


def train(nodes, rollouts, updates, max_norm=1.0, beta=0.8, gamma=0.05, kl=0.01, report=None):
    """`updates` clipped updates on each of `rollouts` draws; returns the mean reward of every draw."""
    history = []
    for r in range(rollouts):
        tokens, keep, advantage, old, reward = nodes.rollout()
        nodes.ref = old  # the reference that the KL term holds to: here the policy that drew the tokens
        for _ in range(updates):
            nodes.gradients(tokens, keep, advantage, old, kl)
            nodes.step(max_norm, beta, gamma)
        history.append(float(reward))
        if report:
            report(r, history[-1], float(nodes.loss.mean()), float(nodes.norms.mean()), nodes.disagreement())
    return history


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--nodes", type=int, default=8)
    ap.add_argument("--rows", type=int, default=64)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--vocab", type=int, default=32)
    ap.add_argument("--rollouts", type=int, default=40)
    ap.add_argument("--updates", type=int, default=4)
    ap.add_argument("--dtype", default="bf16", choices=["bf16", "f32"])
    a = ap.parse_args()
    nodes = Nodes(a.nodes, a.rows, a.width, a.vocab, {"bf16": torch.bfloat16, "f32": torch.float32}[a.dtype])
    print(f"{a.nodes} nodes x {nodes.d} parameters; probability of the right token {nodes.accuracy():.4f}")
    train(nodes, a.rollouts, a.updates, report=lambda r, reward, loss, norm, far: print(
        f"rollout {r:3d}: reward {reward:.3f}  loss {loss:+.4f}  gradient norm {norm:.3f}  disagreement {far:.2e}"))
    print(f"probability of the right token {nodes.accuracy():.4f}")
    assert B.kernel_error() == 0


if __name__ == "__main__":
    main()
