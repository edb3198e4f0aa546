"""Adjustment of logits and its gradient against double precision.  Tolerances, with u = 2^-24: at most eight fp32 roundings (quotient, two
products and differences, bias, 1 / temperature, product) of the magnitudes that enter an element, and the final rounding."""
import numpy as np
import pytest
import torch

from helpers import half_unit, to64

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rand(shape, std, seed, typ="f32"):
    return torch.empty(shape, device=DEV).normal_(0.0, std, generator=_gen(seed)).to(TYPE[typ])


def _case(n, rows, vocab, typ, seed, longest=50, spare_words=0):
    """Everything that an adjustment may be given."""
    count = n * rows
    length = torch.randint(0, longest + 1, (count,), device=DEV, generator=_gen(seed))
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), length.cumsum(0)])
    text = torch.randint(0, max(1, min(vocab, 2 * longest)), (int(start[-1]),), device=DEV, generator=_gen(seed + 1))   # many twice
    text[::7] = torch.tensor([-1, vocab, 2 ** 33, vocab - 1], device=DEV).repeat(text.numel())[:text[::7].numel()]
    words = (vocab + 31) // 32 + spare_words
    allowed = torch.randint(-2 ** 31, 2 ** 31, (n, rows, words), device=DEV, generator=_gen(seed + 2)).int()
    if rows > 2:
        allowed[0, 1], allowed[0, 2] = 0, -1                                 # a row that allows nothing, one that allows all
    one = lambda k, lo, hi: lo + (hi - lo) * torch.rand((n, rows), device=DEV, generator=_gen(seed + k))  # noqa: E731
    return dict(bias=_rand((n, vocab), 1.0, seed + 4), allowed=allowed, history=text, history_start=start, repetition=one(5, 0.8, 1.6),
                frequency=one(6, -0.2, 0.5), presence=one(7, -0.5, 0.5), temperature=one(8, 0.3, 2.0))


def _counts(z, a):
    n, rows, vocab = z.shape
    k, start = a["history"].cpu().numpy(), a["history_start"].cpu().numpy()
    out = np.zeros((n * rows, vocab))
    for r in range(n * rows):
        t = k[start[r]:start[r + 1]]
        np.add.at(out[r], t[(t >= 0) & (t < vocab)], 1)
    return out.reshape(z.shape)


def _forbidden(z, a):
    words, v = a["allowed"].cpu().numpy().view(np.uint32), np.arange(z.shape[2])
    return (words[..., v // 32] >> (v % 32).astype(np.uint32)) & 1 == 0


def _per_row(a, name, default):
    return to64(a[name])[..., None] if a.get(name) is not None else default


def _want(z, a):
    Z = to64(z)
    size = np.abs(Z)
    if a.get("history_start") is not None:
        k, rho = _counts(z, a), _per_row(a, "repetition", 1.0)
        f, p = _per_row(a, "frequency", 0.0) * k, _per_row(a, "presence", 0.0) * (k > 0)
        Z = np.where(k > 0, np.where(Z > 0, Z / rho, Z * rho), Z)
        size = np.abs(Z) + np.abs(f) + np.abs(p)
        Z = Z - f - p
    if a.get("bias") is not None:
        Z, size = Z + to64(a["bias"])[:, None], size + np.abs(to64(a["bias"])[:, None])
    t = _per_row(a, "temperature", 1.0)
    return Z / t, size / t


def _run(z, out=None, **a):
    from paper_2104_11981_b200 import binding as B
    out = torch.full_like(z, float("nan")) if out is None else out
    B.logits_adjust(z, out, **a)
    return out


def _run_grad(d, z, a, out=None):
    from paper_2104_11981_b200 import binding as B
    out = torch.full_like(d, float("nan")) if out is None else out
    rest = {k: a.get(k) for k in ("allowed", "history", "history_start", "repetition", "temperature")}
    B.logits_adjust_grad(d, out, z, **rest)
    return out


def _check(z, typ, a):
    got = to64(_run(z, **a))
    want, size = _want(z, a)
    no = _forbidden(z, a) if a.get("allowed") is not None else np.zeros(z.shape, bool)
    assert np.all(got[no] == -np.inf)
    assert np.all(np.abs(got - want)[~no] <= (8 * U * size + half_unit(typ, want) * (1 + 2.0 ** -10) + 1e-45)[~no])


def _check_grad(d, z, typ, a):
    got, D = to64(_run_grad(d, z, a)), to64(d)
    if a.get("repetition") is not None:
        rho = _per_row(a, "repetition", 1.0)
        D = np.where(_counts(z, a) > 0, np.where(to64(z) > 0, D / rho, D * rho), D)
    want = D / _per_row(a, "temperature", 1.0)
    if a.get("allowed") is not None:
        want = np.where(_forbidden(z, a), 0.0, want)
    assert np.all(np.abs(got - want) <= 8 * U * np.abs(want) + half_unit(typ, want) * (1 + 2.0 ** -10) + 1e-45)


SHAPES = [(1, 1, 1), (1, 1, 31), (2, 3, 33), (3, 5, 1000), (1, 1, 131_072), (2, 2, 50_001), (1, 3, 16_384), (1, 3, 16_385), (2, 4, 8200),
          (300, 2, 64), (1, 500, 4097), (2, 9, 513)]


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("n,rows,vocab", SHAPES)
def test_everything_at_once(n, rows, vocab, typ):
    z, d = _rand((n, rows, vocab), 3.0, vocab, typ), _rand((n, rows, vocab), 1.0, vocab + 1, typ)
    a = _case(n, rows, vocab, typ, vocab, spare_words=vocab % 3)
    _check(z, typ, a)
    _check_grad(d, z, typ, a)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("names", [(), ("bias",), ("allowed",), ("temperature",), ("history", "history_start", "repetition"),
                                   ("history", "history_start", "frequency"), ("history", "history_start", "presence"),
                                   ("history", "history_start"), ("bias", "allowed"), ("allowed", "temperature")])
def test_each_part_alone(names, typ):
    for vocab in (640, 777):
        z, d = _rand((2, 5, vocab), 3.0, 1, typ), _rand((2, 5, vocab), 1.0, 2, typ)
        a = {k: v for k, v in _case(2, 5, vocab, typ, 3).items() if k in names}
        _check(z, typ, a)
        _check_grad(d, z, typ, a)
        if not names:
            assert torch.equal(_run(z), z) and torch.equal(_run_grad(d, None, {}), d)


@pytest.mark.parametrize("longest", [3000, 40_000])
def test_long_texts(longest):
    """Longer than a CTA has threads, most tokens many times; more than 65535 of one."""
    for vocab, typ in ((5000, "f32"), (200, "f32"), (5001, "bf16")):
        z = _rand((1, 3, vocab), 3.0, 1, typ)
        a = _case(1, 3, vocab, typ, 2, longest)
        _check(z, typ, a)
        text = torch.full((70_000,), vocab - 1, device=DEV)
        a.update(history=text, history_start=torch.tensor([0, 70_000, 70_000, 70_000], device=DEV))
        _check(z, typ, a)
        _check_grad(_rand((1, 3, vocab), 3.0, 3, typ), z, typ, a)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_strides_and_alignment(shift, typ):
    n, rows, vocab, ld = 2, 6, 1000, 1024
    z, d = (_rand((n, rows, ld), 2.0, k, typ)[..., shift:shift + vocab] for k in range(2))
    a = _case(n, rows, vocab, typ, 5)
    a["bias"] = _rand((n, vocab + 7), 1.0, 9)[:, 3:vocab + 3]
    for width in (ld, ld + 3):
        out = torch.full((n, rows, width), 9.0, device=DEV, dtype=TYPE[typ])
        view = out[..., shift:shift + vocab]
        for got, want in ((lambda: _run(z, view, **a), _run(z.contiguous(), **a)),
                          (lambda: _run_grad(d, z, a, view), _run_grad(d.contiguous(), z.contiguous(), a))):
            got()
            assert torch.equal(view, want)
            assert bool((torch.cat([out[..., :shift], out[..., shift + vocab:]], -1) == 9.0).all())


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [4096, 50_001])
def test_in_place(vocab, typ):
    z, d, a = _rand((2, 3, vocab), 3.0, 1, typ), _rand((2, 3, vocab), 1.0, 2, typ), _case(2, 3, vocab, typ, 3)
    want = _run(z, **a)
    once = z.clone()
    assert torch.equal(_run(once, once, **a), want)
    grad = _run_grad(d, z, a)
    over = d.clone()
    assert torch.equal(_run_grad(over, z, a, over), grad)
    over = z.clone()
    assert torch.equal(_run_grad(d, over, a, over), grad)


def test_one_mask_for_all_rows():
    z = _rand((2, 5, 300), 1.0, 1)
    mask = torch.randint(-2 ** 31, 2 ** 31, (1, 1, 10), device=DEV, generator=_gen(2)).int()
    wide = mask.expand(2, 5, 10)
    assert wide.stride(0) == 0
    assert torch.equal(_run(z, allowed=wide), _run(z, allowed=wide.contiguous()))


def test_forbidden_places_may_hold_anything():
    """NaN and infinities in logits, gradients and biases where the mask forbids; -inf logits stay -inf."""
    z, d, a = _rand((1, 4, 500), 3.0, 1), _rand((1, 4, 500), 1.0, 2), _case(1, 4, 500, "f32", 3)
    clean, grad = _run(z, **a), _run_grad(d, z, a)
    no = torch.from_numpy(_forbidden(z, a)).to(DEV)
    for bad in (float("nan"), float("inf"), -float("inf")):
        z[no], d[no] = bad, bad
        assert torch.equal(_run(z, **a), clean) and torch.equal(_run_grad(d, z, a), grad)
    z[0, 2, 9], a["allowed"] = -float("inf"), None
    assert float(_run(z, **a)[0, 2, 9]) == -float("inf")


def test_bounds_outside_the_text_are_held():
    """Bounds below 0 or beyond the text's length read nothing there."""
    z, a = _rand((1, 3, 200), 1.0, 1), _case(1, 3, 200, "f32", 3)
    a["history"] = torch.arange(10, device=DEV)
    a["history_start"] = torch.tensor([-5, 4, 2, 1000], device=DEV)
    held = dict(a, history=torch.tensor([0, 1, 2, 3, 2, 3, 4, 5, 6, 7, 8, 9], device=DEV), history_start=torch.tensor([0, 4, 4, 12], device=DEV))
    assert torch.equal(_run(z, **a), _run(z, **held))


def test_no_rows_and_no_text():
    z = torch.empty((2, 0, 100), device=DEV)
    _run(z, bias=_rand((2, 100), 1.0, 1))
    z = _rand((1, 2, 100), 1.0, 1)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    start = torch.zeros(3, dtype=torch.int64, device=DEV)
    a = dict(history=none, history_start=start, repetition=torch.full((1, 2), 2.0, device=DEV))
    assert torch.equal(_run(z, **a), z)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_offsets_beyond_32_bits(typ):
    """More than 2^31 logits: the last rows are those of a short call on them."""
    rows, vocab = 42_000, 51_200
    z = torch.empty((1, rows, vocab), device=DEV, dtype=TYPE[typ])
    z[:, -3:] = _rand((1, 3, vocab), 2.0, 1, typ)
    z[:, :-3] = 1.0
    a = _case(1, 3, vocab, typ, 4)
    long = dict(bias=a["bias"], temperature=torch.ones((1, rows), device=DEV), repetition=torch.ones((1, rows), device=DEV))
    for name in ("temperature", "repetition"):
        long[name][:, -3:] = a[name]
    long["history"] = a["history"]
    long["history_start"] = torch.cat([torch.zeros(rows - 3, dtype=torch.int64, device=DEV), a["history_start"]])
    short = {k: a[k] for k in long}
    want = _run(z[:, -3:].contiguous(), **short)
    assert torch.equal(_run(z, z, **long)[:, -3:], want)


def test_gradient_is_the_slope_of_the_forward_pass():
    """Piecewise linear: differences within a piece are exact to rounding."""
    z, d, a = _rand((1, 4, 90), 3.0, 1), _rand((1, 4, 90), 1.0, 2), _case(1, 4, 90, "f32", 3, longest=90)
    z = torch.where(z.abs() < 0.6, torch.full_like(z, 0.7), z)               # away from the penalty's corner at 0
    grad, no = _run_grad(d, z, a), torch.from_numpy(_forbidden(z, a)).to(DEV)
    for at in ((0, 0, 0), (0, 3, 89), (0, 2, 5), (0, 2, 50), (0, 0, 31)):
        ends = []
        for sign in (0.5, -0.5):
            moved = z.clone()
            moved[at] += sign
            ends.append(float((to64(_run(moved, **a).masked_fill(no, 0.0)) * to64(d)).sum()))
        assert abs(ends[0] - ends[1] - float(grad[at])) <= 2e-4


def test_on_another_stream_and_captured():
    z, a = _rand((2, 3, 6000), 3.0, 1, "bf16"), _case(2, 3, 6000, "bf16", 2)
    want = _run(z, **a)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(z)
    from paper_2104_11981_b200 import binding as B
    B.logits_adjust(z, out, stream=stream, **a)
    stream.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _run(z, out, **a)
    z.mul_(-0.5)
    a["temperature"].add_(1.0)
    graph.replay()
    assert torch.equal(out, _run(z, **a))
