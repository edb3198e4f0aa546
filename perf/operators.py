"""What is measured of the language-model training operators: global gradient norms with clipping,
layer norm in both directions, and the clipped policy loss with its gradient.

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes a case's inputs and `run()`
does one pass: in plain 32-bit torch operations, or (`own`) through this package's binding.  `exact()` gives the
same outputs from the definitions in 64 bits.
"""
import math
import random

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CLIP_EPS = 1e-6     # added to the norm before it divides max_norm
LN_EPS = 1e-5


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # 8 nodes with a 4096-parameter model in a dozen tensors: launches are all there is to pay
        dict(name="clip 8x4k", op="clip", n=8, d=4096, tensors=12, src="f32", dst="f32", align=1, over=1.5),
        # 16 replicas of a 25.6M-parameter model, 161 tensors packed without gaps into the step's fp32 rows
        dict(name="clip 16x25.6M", op="clip", n=16, d=25_557_032, tensors=161, src="f32", dst="f32", align=1, over=2.0),
        # 64 replicas of an 11.7M-parameter model, bf16 gradients, every tensor on an 8-column boundary
        dict(name="clip 64x11.7M bf16", op="clip", n=64, d=11_689_512, tensors=62, src="bf16", dst="bf16", align=8, over=2.0),
        # one token of one model: the form that serving takes
        dict(name="ln 1 token", op="ln", n=1, rows=1, c=4096, type="bf16", bias=True),
        # 8 nodes, 2048 tokens each, bf16 activations
        dict(name="ln 8x2048x4096", op="ln", n=8, rows=2048, c=4096, type="bf16", bias=True),
        # few tokens a node, narrow fp32 rows
        dict(name="ln grad 4x65x768", op="ln_grad", n=4, rows=65, c=768, type="f32", bias=True),
        # the training step's own size
        dict(name="ln grad 8x2048x4096", op="ln_grad", n=8, rows=2048, c=4096, type="bf16", bias=True),
        # odd width, odd row count, no bias
        dict(name="ln grad 3x1021x2047", op="ln_grad", n=3, rows=1021, c=2047, type="f32", bias=False),
        # log-probability of one token under a wide vocabulary, no gradient asked for
        dict(name="policy 1 token", op="policy", n=1, rows=1, vocab=131_072, type="bf16", ref=False, grad=False),
        # short answers on a middling vocabulary
        dict(name="policy 8x128x32k", op="policy", n=8, rows=128, vocab=32_768, type="bf16", ref=True, grad=True),
        # odd vocabulary in fp32
        dict(name="policy 3x111x50001", op="policy", n=3, rows=111, vocab=50_001, type="f32", ref=True, grad=True),
        # 4 nodes, 1024 tokens each, wide vocabulary
        dict(name="policy 4x1024x128k", op="policy", n=4, rows=1024, vocab=131_072, type="bf16", ref=True, grad=True),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["clip", "ln", "ln_grad", "policy"])
    typ = rng.choice(["f32", "bf16"])
    if op == "clip":
        n = _log(rng, 1, 64)
        return dict(op=op, n=n, d=_log(rng, 1000, 400_000_000 // n), tensors=_log(rng, 1, 200), src=typ,
                    dst=rng.choice(["f32", "bf16"]), align=rng.choice([1, 8]), over=rng.choice([0.5, 2.0, 8.0]))
    n = _log(rng, 1, 16)
    if op == "policy":
        vocab = _log(rng, 500, 140_000)
        return dict(op=op, n=n, rows=_log(rng, 1, max(1, 260_000_000 // (n * vocab))), vocab=vocab, type=typ,
                    ref=rng.random() < 0.7, grad=rng.random() < 0.8)
    c = _log(rng, 33, 16_384)
    return dict(op=op, n=n, rows=_log(rng, 1, max(1, 60_000_000 // (n * c))), c=c, type=typ, bias=rng.random() < 0.7)


# ------------------------------------------------------------------------------------------ inputs
def _sizes(case):
    """Sizes of the case's tensors, d in all: a third small vectors, the rest spread over three decades."""
    rng, t = random.Random(case["d"] * 1009 + case["tensors"]), min(case["tensors"], case["d"])
    share = [10 ** rng.uniform(-4, -3) if k % 3 == 2 else 10 ** rng.uniform(-2, 1) for k in range(t)]
    left = case["d"] - t
    sizes = [1 + int(left * s / sum(share)) for s in share]
    sizes[0] += case["d"] - sum(sizes)
    return sizes


def _offsets(case):
    """First column of each tensor, and the row's width."""
    at, offsets, a = 0, [], case["align"]
    for s in _sizes(case):
        offsets.append(at)
        at += -(-s // a) * a
    return offsets, at


def _normal(shape, std, gen, dtype=torch.float32):
    return torch.empty(shape, device=DEVICE).normal_(0.0, std, generator=gen).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    s = dict(case=case)
    n, op = case["n"], case["op"]
    if op == "clip":
        # per-node gradients, one tensor [n, size] for each parameter; the nodes' scales differ, so that some are clipped
        scale = torch.exp(_normal((n, 1), 0.5, gen))
        s["grads"] = [(_normal((n, k), 1e-3, gen) * scale).to(TYPES[case["src"]]) for k in _sizes(case)]
        s["max_norm"] = 1e-3 * math.sqrt(case["d"]) / case["over"]
        s["norms"] = torch.empty(n, device=DEVICE)
        s["offsets"], s["columns"] = _offsets(case)
        # columns between tensors belong to nobody: the program zeroed the stacked gradient once
        s["out"] = torch.zeros((n, s["columns"]), device=DEVICE, dtype=TYPES[case["dst"]])
        if own:
            from paper_2104_11981_b200 import binding as B
            nodes = [[t[i] for t in s["grads"]] for i in range(n)]
            s["list"] = B.gradients_build(nodes, offsets=s["offsets"])
        return s
    if op in ("ln", "ln_grad"):
        rows, c, typ = case["rows"], case["c"], TYPES[case["type"]]
        s["x"] = (_normal((n, rows, c), 1.0, gen) + _normal((n, rows, 1), 0.5, gen)).to(typ)
        # weights and biases are columns of the stacked parameters, one row a node
        s["params"] = _normal((n, 2 * c), 0.1, gen)
        s["w"], s["b"] = s["params"][:, :c], s["params"][:, c:]
        s["w"].add_(1.0)
        s["mean"] = torch.empty((n, rows), device=DEVICE)
        s["rstd"] = torch.empty((n, rows), device=DEVICE)
        s["out"] = torch.empty_like(s["x"])
        if op == "ln_grad":
            s["dy"] = _normal((n, rows, c), 1e-2, gen, typ)
            x = s["x"].double()
            s["mean"].copy_(x.mean(-1))
            s["rstd"].copy_((x.var(-1, unbiased=False) + LN_EPS).rsqrt())
            del x
            s["g"] = torch.zeros((n, 2 * c), device=DEVICE)
            if own:
                from paper_2104_11981_b200 import binding as B
                s["work"] = torch.empty(B.layer_norm_grad_workspace_bytes(n, rows, c), dtype=torch.uint8, device=DEVICE)
        return s
    rows, v = case["rows"], case["vocab"]
    s["logits"] = _normal((n, rows, v), 2.0, gen, TYPES[case["type"]])
    s["tokens"] = torch.randint(0, v, (n, rows), device=DEVICE, generator=gen)
    picked = torch.gather(s["logits"], 2, s["tokens"][..., None])[..., 0].float()
    logp = picked - torch.stack([torch.logsumexp(z.float(), -1) for z in s["logits"]])
    s["lo"], s["hi"], s["kl"] = 0.2, 0.28, 0.05 if case["ref"] else 0.0
    # the objective has corners at these ratios: a token closer than rounding to one has no slope to compare
    moved = _normal((n, rows), 0.2, gen)
    at = torch.exp(-moved)
    corner = ((at - (1.0 - s["lo"])).abs() < 1e-3) | ((at - (1.0 + s["hi"])).abs() < 1e-3)
    s["old"] = logp + moved + 0.01 * corner
    s["ref"] = logp + _normal((n, rows), 0.3, gen) if case["ref"] else None
    s["adv"] = _normal((n, rows), 1.0, gen)
    # a quarter of the tokens belong to prompts and padding; the others share the node's unit weight
    keep = (torch.rand((n, rows), device=DEVICE, generator=gen) >= 0.25).float()
    if rows == 1:
        keep.fill_(1.0)
    s["weight"] = keep / keep.sum(1, keepdim=True).clamp(min=1.0)
    s["loss"] = torch.empty(n, device=DEVICE)
    s["logp"] = torch.empty((n, rows), device=DEVICE)
    s["out"] = torch.empty_like(s["logits"]) if case["grad"] else None
    if own:
        from paper_2104_11981_b200 import binding as B
        s["work"] = torch.empty(B.policy_loss_workspace_bytes(n, rows, v), dtype=torch.uint8, device=DEVICE)
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    return (_run_own if own else _PLAIN[s["case"]["op"]])(s)


def _run_own(s):
    from paper_2104_11981_b200 import binding as B
    op = s["case"]["op"]
    if op == "clip":
        B.gradient_clip(s["list"], s["max_norm"], s["norms"], s["out"])
        return dict(norms=s["norms"], g=s["out"])
    bias = s["b"] if op != "policy" and s["case"]["bias"] else None
    if op == "ln":
        B.layer_norm(s["x"], s["w"], bias, LN_EPS, s["out"], s["mean"], s["rstd"])
        return dict(y=s["out"], mean=s["mean"], rstd=s["rstd"])
    if op == "ln_grad":
        c = s["case"]["c"]
        dw, db = s["g"][:, :c], s["g"][:, c:] if bias is not None else None
        B.layer_norm_grad(s["x"], s["dy"], s["w"], s["mean"], s["rstd"], s["out"], dw, db, s["work"])
        return dict(dx=s["out"], dw=dw, db=db)
    B.policy_loss_grad(s["logits"], s["tokens"], s["weight"], s["adv"], s["old"], s["ref"], s["lo"], s["hi"], s["kl"],
                       s["loss"], s["logp"], s["out"], s["work"])
    return dict(loss=s["loss"], logp=s["logp"], dlogits=s["out"])


def _plain_clip(s):
    ends = s["offsets"][1:] + [s["columns"]]
    g = torch.cat([torch.nn.functional.pad(t.float(), (0, e - o - t.shape[1]))
                   for t, o, e in zip(s["grads"], s["offsets"], ends)], 1)
    norms = (g * g).sum(1).sqrt()
    scale = (s["max_norm"] / (norms + CLIP_EPS)).clamp(max=1.0)
    return dict(norms=norms, g=(g * scale[:, None]).to(s["out"].dtype))


def _plain_ln(s):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    x = x - mean
    rstd = 1.0 / ((x * x).mean(-1, keepdim=True) + LN_EPS).sqrt()
    y = x * rstd * s["w"][:, None]
    if s["case"]["bias"]:
        y = y + s["b"][:, None]
    return dict(y=y.to(s["x"].dtype), mean=mean[..., 0], rstd=rstd[..., 0])


def _plain_ln_grad(s):
    dy, rstd = s["dy"].float(), s["rstd"][..., None]
    xh = (s["x"].float() - s["mean"][..., None]) * rstd
    dw = (dy * xh).sum(1)
    wdy = dy * s["w"][:, None]
    dx = rstd * (wdy - wdy.mean(-1, keepdim=True) - xh * (wdy * xh).mean(-1, keepdim=True))
    return dict(dx=dx.to(s["x"].dtype), dw=dw, db=dy.sum(1) if s["case"]["bias"] else None)


def _plain_policy(s):
    z = s["logits"].float()
    e = z - z.amax(-1, keepdim=True)
    picked = torch.gather(e, 2, s["tokens"][..., None])[..., 0]
    e = e.exp()
    total = e.sum(-1)
    kept = s["weight"] != 0
    logp = torch.where(kept, picked - total.log(), 0.0)
    adv = s["adv"]
    ratio = (logp - s["old"]).exp()
    free, held = ratio * adv, ratio.clamp(1.0 - s["lo"], 1.0 + s["hi"]) * adv
    loss = -torch.minimum(free, held)
    slope = torch.where(free <= held, -free, 0.0)
    if s["ref"] is not None:
        far = s["ref"] - logp
        loss = loss + s["kl"] * (far.exp() - far - 1.0)
        slope = slope + s["kl"] * (1.0 - far.exp())
    loss = torch.where(kept, s["weight"] * loss, 0.0).sum(1)
    if s["out"] is None:
        return dict(loss=loss, logp=logp, dlogits=None)
    slope = torch.where(kept, s["weight"] * slope, 0.0)
    d = e * (-slope / total)[..., None]
    d = d.scatter_add(2, s["tokens"][..., None], slope[..., None])
    return dict(loss=loss, logp=logp, dlogits=d.to(s["logits"].dtype))


_PLAIN = {"clip": _plain_clip, "ln": _plain_ln, "ln_grad": _plain_ln_grad, "policy": _plain_policy}


# ------------------------------------------------------------------------------------------ work and truth
def work(case):
    """Bytes and operations that a pass cannot do without: every input read once, every output written once."""
    n, op = case["n"], case["op"]
    size = {"f32": 4, "bf16": 2}
    if op == "clip":
        e = n * case["d"]
        return dict(bytes=e * size[case["src"]] + n * _offsets(case)[1] * size[case["dst"]] + 4 * n, flops=3 * e)
    k = size[case["type"]]
    if op == "policy":
        r = n * case["rows"]
        e = r * case["vocab"]
        return dict(bytes=e * k * (2 if case["grad"] else 1) + 28 * r, flops=e * (6 if case["grad"] else 4))
    r, c = n * case["rows"], case["c"]
    params = 4 * n * c * (2 if case["bias"] else 1)
    if op == "ln":
        return dict(bytes=2 * r * c * k + 8 * r + params, flops=7 * r * c)
    return dict(bytes=3 * r * c * k + 8 * r + 4 * n * c + params, flops=14 * r * c)


def exact(case, seed):
    """The outputs of run() on prepare()'s inputs, from the definitions in 64 bits, node by node."""
    s = prepare(case, seed)
    nodes = range(case["n"])
    if case["op"] == "clip":
        norms = torch.zeros(case["n"], device=DEVICE, dtype=torch.float64)
        g = torch.zeros((case["n"], s["columns"]), device=DEVICE, dtype=torch.float64)
        for t, o in zip(s["grads"], s["offsets"]):
            g[:, o:o + t.shape[1]] = t
        for i in nodes:
            norms[i] = torch.linalg.vector_norm(g[i])
            g[i] *= min(1.0, s["max_norm"] / (float(norms[i]) + CLIP_EPS))
        return dict(norms=norms, g=g)
    if case["op"] == "ln":
        x = s["x"].double()
        var, mean = torch.var_mean(x, -1, unbiased=False)
        rstd = (var + LN_EPS) ** -0.5
        x.sub_(mean[..., None]).mul_(rstd[..., None]).mul_(s["w"].double()[:, None])
        if case["bias"]:
            x.add_(s["b"].double()[:, None])
        return dict(y=x, mean=mean, rstd=rstd)
    if case["op"] == "ln_grad":
        # the Jacobian of a row applied to w dy: rstd (I - 1 1^T / c - xh xh^T / c), the row's statistics being inputs
        dx, dw, db = [], [], []
        for i in nodes:
            dy, r = s["dy"][i].double(), s["rstd"][i].double()
            xh = (s["x"][i].double() - s["mean"][i].double()[:, None]) * r[:, None]
            v = dy * s["w"][i].double()
            along = torch.einsum("rc,rc->r", v, xh) / case["c"]
            dx.append((v - torch.einsum("rc->r", v)[:, None] / case["c"] - along[:, None] * xh) * r[:, None])
            dw.append(torch.einsum("rc,rc->c", dy, xh))
            db.append(torch.einsum("rc->c", dy))
        return dict(dx=torch.stack(dx), dw=torch.stack(dw), db=torch.stack(db) if case["bias"] else None)
    loss, logps, grads = [], [], []
    for i in nodes:
        logq = torch.log_softmax(s["logits"][i].double(), -1)
        w = s["weight"][i].double()
        lp = torch.where(w != 0, logq[torch.arange(case["rows"], device=DEVICE), s["tokens"][i]], 0.0)
        adv, r = s["adv"][i].double(), torch.exp(lp - s["old"][i].double())
        top = torch.where(adv >= 0, 1.0 + s["hi"], 1.0 - s["lo"])
        inside = torch.where(adv >= 0, r <= top, r >= top)   # the side on which the objective may still be improved
        term, slope = -adv * torch.where(inside, r, top), -adv * r * inside
        if s["ref"] is not None:
            u = torch.exp(s["ref"][i].double() - lp)
            term = term + s["kl"] * (u - torch.log(u) - 1.0)
            slope = slope + s["kl"] * (1.0 - u)
        loss.append((w * term).sum())
        logps.append(lp)
        if case["grad"]:
            d = logq.exp_().mul_(-(w * slope)[:, None])
            d[torch.arange(case["rows"], device=DEVICE), s["tokens"][i]] += w * slope
            grads.append(d)
    return dict(loss=torch.stack(loss), logp=torch.stack(logps), dlogits=torch.stack(grads) if case["grad"] else None)
