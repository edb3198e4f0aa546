"""The training operators together, as examples/policy_finetune.py runs them: gradients against automatic differentiation
in double precision, and a short training run."""
import os
import sys

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
pytestmark = pytest.mark.gpu


def test_gradients_match_automatic_differentiation():
    """fp32 throughout.  The products add up to `vocab` or `rows` fp32 terms, whose error grows like the root of their number:
    1e-5 of a gradient's norm is some fifty roundings."""
    from policy_finetune import Nodes
    nodes = Nodes(n=3, rows=21, width=40, vocab=77, dtype=torch.float32, seed=4)
    nodes.x.add_(torch.empty_like(nodes.x).normal_(0.0, 0.05, generator=nodes.gen))     # replicas differ
    tokens, keep, advantage, old, _ = nodes.rollout()
    old = old + torch.empty_like(old).normal_(0.0, 0.3, generator=nodes.gen)
    nodes.ref = old + torch.empty_like(old).normal_(0.0, 0.3, generator=nodes.gen)
    keep[:, ::4] = 0.0
    nodes.gradients(tokens, keep, advantage, old, 0.1)
    got, loss = [nodes.dweight, nodes.dbias, nodes.dhead], nodes.loss.double()
    w, n = nodes.width, nodes.n
    x = nodes.x.double()
    ps = [x[:, :w].clone(), x[:, w:2 * w].clone(), x[:, 2 * w:].reshape(n, nodes.vocab, w).clone()]
    for p in ps:
        p.requires_grad_(True)
    h = nodes.hidden.double()
    mu, var = h.mean(-1, keepdim=True), h.var(-1, unbiased=False, keepdim=True)
    y = (h - mu) / torch.sqrt(var + 1e-5) * ps[0][:, None] + ps[1][:, None]
    lp = torch.log_softmax(y @ ps[2].transpose(1, 2), -1).gather(2, tokens[..., None])[..., 0]
    r = torch.exp(lp - old.double())
    far = nodes.ref.double() - lp
    obj = torch.minimum(r * advantage.double(), r.clamp(0.8, float(np.float32(1.0) + np.float32(0.28))) * advantage.double())
    want = (keep.double() * (-obj + float(np.float32(0.1)) * (torch.exp(far) - far - 1))).sum(1)
    want.sum().backward()
    want = want.detach()
    assert float((loss - want).abs().max()) <= 1e-5 * float(want.abs().max() + 1)
    for g, p in zip(got, ps):
        assert float((g.double() - p.grad).norm() / p.grad.norm()) <= 1e-5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_run_learns(dtype):
    from paper_2104_11981_b200 import binding as B
    from policy_finetune import Nodes, train
    nodes = Nodes(n=8, rows=64, width=128, vocab=32, dtype=dtype, seed=1)
    before = nodes.accuracy()
    rewards = train(nodes, rollouts=30, updates=4)
    after = nodes.accuracy()
    assert np.isfinite(rewards).all() and torch.isfinite(nodes.x).all() and B.kernel_error() == 0
    assert before < 0.06 and after > 3 * before and np.mean(rewards[-5:]) > 2 * np.mean(rewards[:3])
    assert nodes.disagreement() < 0.2                       # the replicas learn one policy between them
    assert float(nodes.norms.max()) < 1e4
