"""What is measured of the operators between a replica's tokens and its logits: the embedding and its gradient, the
root-mean-square norm with residual (16, 32 and 8 bits out) and its gradient, dropout, and the adjustment of logits by
penalties, biases, masks and temperature with its gradient.

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes a case's inputs and `run()`
does one pass: in plain 32-bit torch operations, or (`own`) through this package's binding.  `exact()` gives the
same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the token just drawn, in one model: the form that serving takes
        dict(name="embed 1 token", op="embed", n=1, rows=1, vocab=131_072, c=4096, table="f32", type="bf16"),
        # 8 nodes, 2048 tokens each: what a training step begins with
        dict(name="embed 8x2048", op="embed", n=8, rows=2048, vocab=32_768, c=1024, table="f32", type="bf16"),
        # and what it ends with: the whole table's gradient, into the fp32 rows that the update rules read
        dict(name="embed grad 8x2048", op="embed_grad", n=8, rows=2048, vocab=32_768, c=1024, grad="f32", type="bf16"),
        # many tokens, odd width and vocabulary
        dict(name="embed grad 2x20011", op="embed_grad", n=2, rows=20_011, vocab=50_001, c=1001, grad="bf16", type="f32"),
        # one token of one model, 8-bit output for the product behind it
        dict(name="rms 1 token e4m3", op="rms", n=1, rows=1, c=4096, type="bf16", residual=True, out="e4m3"),
        # 8 nodes, 2048 tokens each, residual stream
        dict(name="rms 8x2048x4096", op="rms", n=8, rows=2048, c=4096, type="bf16", residual=True, out="same"),
        # odd width, odd row count, no gradient from the residual stream
        dict(name="rms grad 3x1021x2047", op="rms_grad", n=3, rows=1021, c=2047, type="f32", residual=False),
        # the training step's own size
        dict(name="rms grad 8x2048x4096", op="rms_grad", n=8, rows=2048, c=4096, type="bf16", residual=True),
        # a small fp32 model's activations
        dict(name="dropout 4x65x769", op="dropout", n=4, rows=65, c=769, type="f32", residual=False, p=0.1),
        # dropout of a branch's output, added to the residual stream
        dict(name="dropout 8x2048x4096", op="dropout", n=8, rows=2048, c=4096, type="bf16", residual=True, p=0.1),
        # one token to be drawn under a wide vocabulary, after a long text and under a grammar
        dict(name="logits 1 token", op="logits", n=1, rows=1, vocab=131_072, type="bf16", history=2048, bias=True, mask=True),
        # a rollout's scores under a middling odd vocabulary, and the way back to the head
        dict(name="logits grad 4x1024x50001", op="logits_grad", n=4, rows=1024, vocab=50_001, type="bf16", history=512, bias=False, mask=True),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "rms", "rms_grad", "dropout", "logits", "logits_grad"])
    typ, n = rng.choice(["f32", "bf16"]), _log(rng, 1, 16)
    if op in ("embed", "embed_grad"):
        c = _log(rng, 33, 8192)
        vocab = _log(rng, 300, max(301, min(140_000, 200_000_000 // (n * c))))
        rows = _log(rng, 1, max(1, min(50_000, 16_000_000 // (n * c))))
        if op == "embed":
            return dict(op=op, n=n, rows=rows, vocab=vocab, c=c, table=rng.choice(["f32", "f32", "bf16"]), type=typ)
        return dict(op=op, n=n, rows=rows, vocab=vocab, c=c, grad=rng.choice(["f32", "bf16"]), type=typ)
    if op in ("logits", "logits_grad"):
        vocab = _log(rng, 500, 140_000)
        return dict(op=op, n=n, rows=_log(rng, 1, max(1, 200_000_000 // (n * vocab))), vocab=vocab, type=typ,
                    history=rng.choice([0, 1, 1]) * _log(rng, 8, 4096), bias=rng.random() < 0.5, mask=rng.random() < 0.7)
    c = _log(rng, 33, 16_384)
    case = dict(op=op, n=n, rows=_log(rng, 1, max(1, 60_000_000 // (n * c))), c=c, type=typ, residual=rng.random() < 0.7)
    if op == "rms":
        case["out"] = rng.choice(["same", "same", "e4m3"])
    if op == "dropout":
        case["p"] = rng.choice([0.05, 0.1, 0.25, 0.5])
    return case


# ------------------------------------------------------------------------------------------ inputs
def _normal(shape, std, gen, dtype=torch.float32):
    return torch.empty(shape, device=DEVICE).normal_(0.0, std, generator=gen).to(dtype)


def _zipf(shape, vocab, gen):
    """Tokens of a text: the k-th commonest with probability log((k + 2) / (k + 1)) / log(vocab + 1)."""
    u = torch.rand(shape, device=DEVICE, generator=gen, dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1)) - 1.0).long().clamp_(0, vocab - 1)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    s = dict(case=case)
    n, rows, op = case["n"], case["rows"], case["op"]
    typ = TYPES[case["type"]]
    if op in ("embed", "embed_grad"):
        c, vocab = case["c"], case["vocab"]
        s["tokens"] = _zipf((n, rows), vocab, gen)
        s["scale"] = math.sqrt(c)
        if op == "embed":
            # the table is a column range of the stacked parameters, one row a node
            s["params"] = _normal((n, vocab * c), 0.02, gen, TYPES[case["table"]])
            s["table"] = s["params"].view(n, vocab, c)
            s["out"] = torch.empty((n, rows, c), device=DEVICE, dtype=typ)
            return s
        s["dy"] = _normal((n, rows, c), 1e-2, gen, typ)
        # and so is its gradient
        s["g"] = torch.zeros((n, vocab * c), device=DEVICE, dtype=TYPES[case["grad"]])
        if own:
            from paper_2104_11981_b200 import binding as B
            s["work"] = torch.empty(B.embedding_grad_workspace_bytes(n, rows, vocab, c), dtype=torch.uint8, device=DEVICE)
        return s
    if op in ("logits", "logits_grad"):
        vocab, count = case["vocab"], n * rows
        s["logits"] = _normal((n, rows, vocab), 2.0, gen, typ)
        if op == "logits_grad":
            s["dout"] = _normal((n, rows, vocab), 1e-3, gen, typ)
        s["out"] = torch.empty_like(s["logits"])
        s["temperature"] = 0.5 + torch.rand((n, rows), device=DEVICE, generator=gen)
        s["bias"] = _normal((n, vocab), 1.0, gen) if case["bias"] else None
        for name in ("history", "start", "repetition", "frequency", "presence", "allowed"):
            s[name] = None
        if case["history"]:
            # rows are at different places of their texts
            length = torch.randint(case["history"] // 2, case["history"] + 1, (count,), device=DEVICE, generator=gen)
            s["start"] = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEVICE), length.cumsum(0)])
            s["total"] = int(s["start"][-1])
            s["history"] = _zipf((s["total"],), vocab, gen)
            s["repetition"] = 1.0 + 0.3 * torch.rand((n, rows), device=DEVICE, generator=gen)
            s["frequency"] = 0.1 * torch.rand((n, rows), device=DEVICE, generator=gen)
            s["presence"] = 0.5 * torch.rand((n, rows), device=DEVICE, generator=gen)
        if case["mask"]:
            # a bit a token: half of the rows are free, a quarter allows every other token, a quarter a sixteenth of them
            words = [torch.randint(-2 ** 31, 2 ** 31, (n, rows, (vocab + 31) // 32), device=DEVICE, generator=gen).int() for _ in range(4)]
            kind = torch.randint(0, 4, (n, rows, 1), device=DEVICE, generator=gen)
            few = words[0] & words[1] & words[2] & words[3]
            s["allowed"] = torch.where(kind < 2, torch.full_like(few, -1), torch.where(kind == 2, words[0], few))
        return s
    c = case["c"]
    s["x"] = _normal((n, rows, c), 1.0, gen, typ)
    s["residual"] = _normal((n, rows, c), 1.5, gen, typ) if case["residual"] else None
    s["out"] = torch.empty_like(s["x"])
    if op == "dropout":
        # seed and step of the training run, where captured steps find them
        s["state"] = torch.randint(0, 2 ** 62, (2,), device=DEVICE, generator=gen)
        s["site"] = 3
        return s
    s["params"] = _normal((n, c), 0.1, gen)
    s["w"] = s["params"].add_(1.0)
    s["rstd"] = torch.empty((n, rows), device=DEVICE)
    if op == "rms":
        s["h"] = torch.empty_like(s["x"]) if case["residual"] else None
        if case["out"] == "e4m3":
            s["out"] = torch.empty((n, rows, c), device=DEVICE, dtype=torch.float8_e4m3fn)
            s["scales"] = torch.empty((n, rows), device=DEVICE)
        return s
    s["dy"] = _normal((n, rows, c), 1e-2, gen, typ)
    s["rstd"].copy_((s["x"].double().square().mean(-1) + EPS).rsqrt())
    if case["residual"]:
        s["residual"] = _normal((n, rows, c), 1e-2, gen, typ)   # the gradient that comes along the residual stream
    s["g"] = torch.zeros((n, c), device=DEVICE)
    if own:
        from paper_2104_11981_b200 import binding as B
        s["work"] = torch.empty(B.rms_norm_grad_workspace_bytes(n, rows, c), dtype=torch.uint8, device=DEVICE)
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    return (_OWN if own else _PLAIN)[s["case"]["op"]](s)


def _own_embed(s):
    from paper_2104_11981_b200 import binding as B
    B.embedding(s["table"], s["tokens"], s["out"], s["scale"])
    return s["out"]


def _own_embed_grad(s):
    from paper_2104_11981_b200 import binding as B
    case = s["case"]
    B.embedding_grad(s["tokens"], s["dy"], s["g"].view(case["n"], case["vocab"], case["c"]), s["work"], s["scale"])
    return s["g"]


def _own_rms(s):
    from paper_2104_11981_b200 import binding as B
    if s["case"]["out"] == "e4m3":
        B.rms_norm(s["x"], s["w"], EPS, None, s["rstd"], s["residual"], s["h"], s["out"], s["scales"])
        return dict(h=s["h"], rstd=s["rstd"], q=s["out"], scales=s["scales"])
    B.rms_norm(s["x"], s["w"], EPS, s["out"], s["rstd"], s["residual"], s["h"])
    return dict(y=s["out"], h=s["h"], rstd=s["rstd"])


def _own_rms_grad(s):
    from paper_2104_11981_b200 import binding as B
    B.rms_norm_grad(s["x"], s["dy"], s["w"], s["rstd"], s["out"], s["g"], s["work"], s["residual"])
    return dict(dh=s["out"], dw=s["g"])


def _own_dropout(s):
    from paper_2104_11981_b200 import binding as B
    B.dropout(s["x"], s["case"]["p"], s["state"], s["out"], s["site"], s["residual"])
    return s["out"]


def _own_logits(s):
    from paper_2104_11981_b200 import binding as B
    B.logits_adjust(s["logits"], s["out"], s["bias"], s["allowed"], s["history"], s["start"], s["repetition"], s["frequency"],
                    s["presence"], s["temperature"])
    return s["out"]


def _own_logits_grad(s):
    from paper_2104_11981_b200 import binding as B
    B.logits_adjust_grad(s["dout"], s["out"], s["logits"], s["allowed"], s["history"], s["start"], s["repetition"], s["temperature"])
    return s["out"]


_OWN = {"embed": _own_embed, "embed_grad": _own_embed_grad, "rms": _own_rms, "rms_grad": _own_rms_grad,
        "dropout": _own_dropout, "logits": _own_logits, "logits_grad": _own_logits_grad}


def _flat_tokens(s):
    case = s["case"]
    return (s["tokens"] + torch.arange(case["n"], device=DEVICE)[:, None] * case["vocab"]).reshape(-1)


def _plain_embed(s):
    case = s["case"]
    rows = s["table"].reshape(case["n"] * case["vocab"], case["c"])[_flat_tokens(s)]
    return (rows.float() * s["scale"]).to(s["out"].dtype).reshape(s["out"].shape)


def _plain_embed_grad(s):
    case = s["case"]
    total = torch.zeros((case["n"] * case["vocab"], case["c"]), device=DEVICE)
    total.index_add_(0, _flat_tokens(s), s["dy"].reshape(-1, case["c"]).float())
    return (total * s["scale"]).to(s["g"].dtype).reshape(s["g"].shape)


def _plain_rms(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    rstd = 1.0 / ((h * h).mean(-1, keepdim=True) + EPS).sqrt()
    kept = h.to(s["x"].dtype) if s["residual"] is not None else None
    if s["case"]["out"] == "same":
        return dict(y=(h * rstd * s["w"][:, None]).to(s["x"].dtype), h=kept, rstd=rstd[..., 0])
    v = h * s["w"][:, None]
    top = v.abs().amax(-1, keepdim=True)
    q = (v * (E4M3_MAX / top)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return dict(h=kept, rstd=rstd[..., 0], q=q, scales=(top * rstd / E4M3_MAX)[..., 0])


def _plain_rms_grad(s):
    h, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][..., None]
    xh = h * rstd
    v = dy * s["w"][:, None]
    dh = rstd * (v - xh * (v * xh).mean(-1, keepdim=True))
    if s["residual"] is not None:
        dh = dh + s["residual"].float()
    return dict(dh=dh.to(s["x"].dtype), dw=(dy * xh).sum(1))


def _plain_dropout(s):
    x, p = s["x"], s["case"]["p"]
    limit = int(math.floor(p * 65536.0 + 0.5))
    count = x.numel()
    low = 0xFFFFFFFF
    group = torch.arange((count + 7) // 8, device=DEVICE)
    key0, key1 = s["state"][0] & low, (s["state"][0] >> 32) & low
    a, b, c, d = group & low, group >> 32, (s["state"][1] & low).expand_as(group), torch.full_like(group, s["site"])
    for k in range(10):     # Philox4x32-10; a product's 64 bits are right whatever their sign
        u, v = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = ((v >> 32) & low) ^ b ^ key0, v & low, ((u >> 32) & low) ^ d ^ key1, u & low
        key0, key1 = (key0 + 0x9E3779B9) & low, (key1 + 0xBB67AE85) & low
    bits = torch.stack([a, b, c, d], 1)
    bits = torch.stack([bits & 0xFFFF, bits >> 16], 2).reshape(-1)[:count].reshape(x.shape)
    y = torch.where(bits >= limit, x.float() * (65536.0 / (65536 - limit)), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(x.dtype)


def _plain_counts(s):
    """How often each row's text has each token."""
    case = s["case"]
    count = case["n"] * case["rows"]
    row = torch.repeat_interleave(torch.arange(count, device=DEVICE), s["start"].diff(), output_size=s["total"])
    counts = torch.zeros(count * case["vocab"], device=DEVICE)
    counts.index_add_(0, row * case["vocab"] + s["history"], torch.ones(s["total"], device=DEVICE))
    return counts.reshape(s["logits"].shape)


def _plain_forbidden(s):
    bit = (s["allowed"][..., None] >> torch.arange(32, device=DEVICE, dtype=torch.int32)) & 1
    return bit.reshape(*s["allowed"].shape[:2], -1)[..., :s["case"]["vocab"]] == 0


def _plain_logits(s):
    z = s["logits"].float()
    if s["history"] is not None:
        counts, rep = _plain_counts(s), s["repetition"][..., None]
        z = torch.where(counts > 0, torch.where(z > 0, z / rep, z * rep), z)
        z = z - s["frequency"][..., None] * counts - torch.where(counts > 0, s["presence"][..., None], 0.0)
    if s["bias"] is not None:
        z = z + s["bias"][:, None]
    z = z / s["temperature"][..., None]
    if s["allowed"] is not None:
        z = torch.where(_plain_forbidden(s), -math.inf, z)
    return z.to(s["logits"].dtype)


def _plain_logits_grad(s):
    d = s["dout"].float() / s["temperature"][..., None]
    if s["history"] is not None:
        rep = s["repetition"][..., None]
        d = torch.where(_plain_counts(s) > 0, torch.where(s["logits"] > 0, d / rep, d * rep), d)
    if s["allowed"] is not None:
        d = torch.where(_plain_forbidden(s), 0.0, d)
    return d.to(s["dout"].dtype)


_PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "rms": _plain_rms, "rms_grad": _plain_rms_grad,
          "dropout": _plain_dropout, "logits": _plain_logits, "logits_grad": _plain_logits_grad}


# ------------------------------------------------------------------------------------------ work and truth
def _distinct(rows, vocab):
    """Distinct tokens that are to be expected of a node's text."""
    k = torch.arange(vocab, dtype=torch.float64)
    p = torch.log((k + 2) / (k + 1)) / math.log(vocab + 1)
    return float((1.0 - (1.0 - p) ** rows).sum())


def work(case):
    """Bytes and operations that a pass cannot do without: every input read once, every output written once."""
    n, r, op = case["n"], case["n"] * case["rows"], case["op"]
    size = {"f32": 4, "bf16": 2}
    k = size[case["type"]]
    if op == "embed":
        c = case["c"]
        return dict(bytes=n * _distinct(case["rows"], case["vocab"]) * c * size[case["table"]] + r * (c * k + 8), flops=r * c)
    if op == "embed_grad":
        c = case["c"]
        return dict(bytes=n * case["vocab"] * c * size[case["grad"]] + r * (c * k + 8), flops=r * c)
    if op in ("logits", "logits_grad"):
        e = r * case["vocab"]
        more = (4 * n * case["vocab"] if case["bias"] else 0) + (e / 8 if case["mask"] else 0) + r * (0.75 * case["history"] * 8 + 20)
        return dict(bytes=2 * e * k + more, flops=e * 3)
    e = r * case["c"]
    if op == "dropout":
        return dict(bytes=e * k * (3 if case["residual"] else 2), flops=e * 12)
    if op == "rms":
        out = e + 4 * r if case["out"] == "e4m3" else e * k
        return dict(bytes=e * k * (3 if case["residual"] else 1) + out + 4 * r + 4 * n * case["c"], flops=6 * e)
    return dict(bytes=e * k * (4 if case["residual"] else 3) + 4 * r + 8 * n * case["c"], flops=11 * e)


def _exact_kept(case, s):
    """Which elements dropout keeps, from the generator's definition with products by 16-bit halves."""
    def wide(m, v):     # high and low words of a 32 x 32-bit product
        ml, mh, vl, vh = m & 0xFFFF, m >> 16, v & 0xFFFF, v >> 16
        mid = mh * vl + (ml * vl >> 16)
        top = ml * vh + (mid & 0xFFFF)
        return mh * vh + (mid >> 16) + (top >> 16), (top & 0xFFFF) << 16 | (ml * vl & 0xFFFF)

    seed, step = (int(v) % 2 ** 64 for v in s["state"].tolist())
    groups = -(-s["x"].numel() // 8)
    index = torch.arange(groups, device=DEVICE)
    word = [index % 2 ** 32, index // 2 ** 32, torch.full_like(index, step % 2 ** 32), torch.full_like(index, s["site"])]
    for k in range(10):
        keys = [(seed % 2 ** 32 + k * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + k * 0xBB67AE85) % 2 ** 32]
        (h0, l0), (h1, l1) = wide(0xD2511F53, word[0]), wide(0xCD9E8D57, word[2])
        word = [h1 ^ word[1] ^ keys[0], l1, h0 ^ word[3] ^ keys[1], l0]
    limit = round(case["p"] * 65536)
    kept = torch.empty((groups, 8), dtype=torch.bool, device=DEVICE)
    for j in range(8):
        kept[:, j] = (word[j // 2] // 2 ** (16 * (j % 2))) % 65536 >= limit
    return kept.view(-1)[:s["x"].numel()].view(s["x"].shape), 65536 / (65536 - limit)


def exact(case, seed):
    """The outputs of run() on prepare()'s inputs, from the definitions in 64 bits, node by node."""
    s = prepare(case, seed)
    op, nodes = case["op"], range(case["n"])
    if op == "embed":
        return torch.stack([s["table"][i].index_select(0, s["tokens"][i]).double() * s["scale"] for i in nodes])
    if op == "embed_grad":
        table = []
        for i in nodes:
            order = torch.argsort(s["tokens"][i], stable=True)
            found, length = torch.unique_consecutive(s["tokens"][i][order], return_counts=True)
            g = torch.zeros((case["vocab"], case["c"]), device=DEVICE, dtype=torch.float64)
            g[found] = torch.segment_reduce(s["dy"][i].double()[order], "sum", lengths=length, axis=0) * s["scale"]
            table.append(g.reshape(-1))
        return torch.stack(table)
    if op == "dropout":
        kept, scale = _exact_kept(case, s)
        y = torch.zeros(s["x"].shape, device=DEVICE, dtype=torch.float64)
        y[kept] = s["x"][kept].double() * scale
        return y if s["residual"] is None else y.add_(s["residual"])
    if op == "rms":
        h = s["x"].double() if s["residual"] is None else s["x"].double().add_(s["residual"])
        rstd = (torch.einsum("nrc,nrc->nr", h, h) / case["c"] + EPS) ** -0.5
        kept = None if s["residual"] is None else h.clone()
        y = h.mul_(rstd[..., None]).mul_(s["w"].double()[:, None])
        if case["out"] == "same":
            return dict(y=y, h=kept, rstd=rstd)
        scales = torch.linalg.vector_norm(y, math.inf, -1) / E4M3_MAX
        return dict(h=kept, rstd=rstd, q=y / scales[..., None], scales=scales)
    if op == "rms_grad":
        # the Jacobian of a row applied to w dy: rstd (I - xh xh^T / c), the row's statistic being an input
        dh, dw = [], []
        for i in nodes:
            dy, r = s["dy"][i].double(), s["rstd"][i].double()[:, None]
            xh, v = s["x"][i].double() * r, dy * s["w"][i].double()
            d = r * (v - torch.einsum("rc,rc->r", v, xh)[:, None] / case["c"] * xh)
            dh.append(d if s["residual"] is None else d + s["residual"][i].double())
            dw.append(torch.einsum("rc,rc->c", dy, xh))
        return dict(dh=torch.stack(dh), dw=torch.stack(dw))
    out, rows = [], case["rows"]
    for i in nodes:
        z = (s["logits"][i] if op == "logits" else s["dout"][i]).double()
        t = s["temperature"][i].double()[:, None]
        if s["history"] is not None:
            start = s["start"][i * rows:(i + 1) * rows + 1]
            text = s["history"][int(start[0]):int(start[-1])]
            row = torch.searchsorted(start - start[0], torch.arange(text.numel(), device=DEVICE), right=True) - 1
            places, times = torch.unique(row * case["vocab"] + text, return_counts=True)
            row, token = places // case["vocab"], places % case["vocab"]
            rep, old = s["repetition"][i].double()[row], z[row, token]
            factor = torch.where(s["logits"][i][row, token] > 0, 1.0 / rep, rep)
            if op == "logits":
                z[row, token] = old * factor - s["frequency"][i].double()[row] * times - s["presence"][i].double()[row]
            else:
                z[row, token] = old * factor
        if op == "logits" and s["bias"] is not None:
            z += s["bias"][i].double()
        z /= t
        if s["allowed"] is not None:
            at = torch.arange(case["vocab"], device=DEVICE)
            bit = torch.bitwise_right_shift(s["allowed"][i][:, at // 32], (at % 32).int()) & 1
            z[bit == 0] = -math.inf if op == "logits" else 0.0
        out.append(z)
    return torch.stack(out)
