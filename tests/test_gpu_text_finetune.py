"""The operators between tokens and logits together, as examples/policy_finetune.py --text runs them: gradients against automatic
differentiation in double precision, a short run, and the whole update captured into a graph."""
import os
import sys

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
pytestmark = pytest.mark.gpu


def _nodes(dtype=torch.float32, **kw):
    from policy_finetune import TextNodes
    nodes = TextNodes(**{**dict(n=3, rows=21, width=40, vocab=77, dtype=dtype, seed=4), **kw})
    nodes.x.add_(torch.empty_like(nodes.x).normal_(0.0, 0.05, generator=nodes.gen))     # replicas differ
    return nodes


def test_gradients_match_automatic_differentiation():
    """fp32 throughout.  The products add up to `vocab` or `rows` fp32 terms, whose error grows like the root of their number:
    2e-5 of a gradient's norm is some hundred roundings."""
    from paper_2104_11981_b200 import binding as B
    nodes = _nodes()
    tokens, keep, advantage, old, _ = nodes.rollout()
    old = old + torch.empty_like(old).normal_(0.0, 0.3, generator=nodes.gen)
    nodes.ref = old + torch.empty_like(old).normal_(0.0, 0.3, generator=nodes.gen)
    keep[:, ::4] = 0.0
    nodes.state[1] = 5
    nodes.gradients(tokens, keep, advantage, old, 0.1)
    got, loss = [nodes.dtable, nodes.dlayer, nodes.dweight, nodes.dhead], nodes.loss.double()
    ones = torch.ones_like(nodes.h)
    mask = torch.empty_like(ones)
    B.dropout(ones, nodes.P_DROP, nodes.state, mask)                          # mask and scale in one
    assert 0.02 < float((mask == 0).double().mean()) < 0.25
    n, w, v, at, x = nodes.n, nodes.width, nodes.vocab, nodes.at, nodes.x.double()
    ps = [x[:, :at[1]].reshape(n, v, w).clone(), x[:, at[1]:at[2]].reshape(n, w, w).clone(), x[:, at[2]:at[3]].clone(), x[:, at[3]:].reshape(n, v, w).clone()]
    for p in ps:
        p.requires_grad_(True)
    e = torch.stack([ps[0][i][nodes.context[i]] for i in range(n)]) * float(np.float32(w ** 0.5))
    h = e + (e @ ps[1].transpose(1, 2)) * mask.double()
    y = h * (h.square().mean(-1, keepdim=True) + float(np.float32(1e-5))).rsqrt() * ps[2][:, None]
    z = y @ ps[3].transpose(1, 2)
    rep = float(np.float32(1.2))
    context = torch.zeros(z.shape, dtype=torch.bool, device=z.device).scatter_(2, nodes.context[..., None], True)
    z = torch.where(context, torch.where(z > 0, z / rep, z * rep), z) / float(np.float32(nodes.TEMPERATURE))
    bits = (nodes.allowed[..., None] >> torch.arange(32, device=z.device, dtype=torch.int32)) & 1
    z = z.masked_fill(bits.flatten(2)[..., :v] == 0, -float("inf"))
    lp = torch.log_softmax(z, -1).gather(2, tokens[..., None])[..., 0]
    r = torch.exp(lp - old.double())
    far = nodes.ref.double() - lp
    obj = torch.minimum(r * advantage.double(), r.clamp(0.8, float(np.float32(1.0) + np.float32(0.28))) * advantage.double())
    want = (keep.double() * (-obj + float(np.float32(0.1)) * (torch.exp(far) - far - 1))).sum(1)
    want.sum().backward()
    want = want.detach()
    assert float((loss - want).abs().max()) <= 2e-5 * float(want.abs().max() + 1)
    for g, p in zip(got, ps):
        assert float((g.double() - p.grad).norm() / p.grad.norm()) <= 2e-5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_short_run(dtype):
    """Runs, stays finite, and only allowed tokens are drawn."""
    from paper_2104_11981_b200 import binding as B
    from policy_finetune import train
    nodes = _nodes(dtype, n=8, rows=64, width=64, vocab=32)
    rewards = train(nodes, rollouts=6, updates=2)
    tokens = nodes.rollout()[0]
    bits = (torch.gather(nodes.allowed, 2, (tokens // 32)[..., None])[..., 0] >> (tokens % 32)) & 1
    assert bool((bits == 1).all())
    assert np.isfinite(rewards).all() and torch.isfinite(nodes.x).all() and B.kernel_error() == 0
    assert int(nodes.state[1]) == 12 and nodes.disagreement() < 1.0


def test_an_update_captured_into_a_graph():
    """Replays of one captured update give the eager updates' parameters, each with a mask of its own."""
    a, b = _nodes(torch.bfloat16), _nodes(torch.bfloat16)
    assert torch.equal(a.x, b.x)
    tokens, keep, advantage, old, _ = a.rollout()
    for nodes in (a, b):
        nodes.ref = old

    def update(nodes):
        nodes.gradients(tokens, keep, advantage, old, 0.01)
        nodes.step(1.0, 0.8, 0.05)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        update(b)
    torch.cuda.current_stream().wait_stream(side)
    update(a)
    assert torch.equal(a.x, b.x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        update(b)
    for _ in range(3):
        update(a)
        graph.replay()
        assert torch.equal(a.x, b.x) and torch.equal(a.g, b.g)
