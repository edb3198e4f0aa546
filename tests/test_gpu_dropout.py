"""Dropout: the mask bit by bit against the documented generator, the values against double precision (a product and an addition: two units
in the last place of fp32 of the magnitudes that enter, and the final rounding)."""
import numpy as np
import pytest
import torch

from helpers import half_unit, to64
from helpers_philox import kept

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rand(shape, std, seed, typ="f32"):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, device=DEV).normal_(0.0, std, generator=g).to(TYPE[typ])


def _state(seed, step):
    return torch.tensor([seed, step], dtype=torch.int64, device=DEV)


def _run(x, p, state, site=0, r=None, y=None):
    from paper_2104_11981_b200 import binding as B
    y = torch.full_like(x, float("nan")) if y is None else y
    B.dropout(x, p, state, y, site, r)
    return y


def _check(x, typ, p, seed, step, site, r=None):
    y = _run(x, p, _state(seed, step), site, r)
    keep, scale = kept(0, x.numel(), p, seed, step, site)
    X, R = to64(x), to64(r) if r is not None else 0.0
    want = np.where(keep.reshape(X.shape), X * scale, 0.0) + R
    tol = 2 * U * (np.abs(X * scale) + np.abs(R)) + half_unit(typ, want) * (1 + 2.0 ** -10) + 1e-45
    assert np.all(np.abs(to64(y) - want) <= tol)
    dropped = ~keep.reshape(X.shape)
    assert np.array_equal(to64(y)[dropped], (R + np.zeros_like(X))[dropped])
    return y


SHAPES = [(1, 1, 1), (1, 1, 7), (1, 1, 8), (2, 3, 5), (1, 1, 4096), (4, 65, 769), (3, 11, 33), (2, 100, 1024), (1, 700, 40), (5, 1, 24),
          (1, 3, 100_003), (300, 2, 16), (1, 5000, 3)]


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_masks_and_values(shape, typ):
    x, r = _rand(shape, 1.0, 1, typ), _rand(shape, 1.0, 2, typ)
    for p, seed, step, site in ((0.1, 0, 0, 0), (0.5, 2 ** 62 + 12345, 2 ** 33 + 7, 2 ** 32 - 1), (0.999, -1, 1, 5)):
        _check(x, typ, p, seed, step, site)
        _check(x, typ, p, seed, step, site, r)


def test_probabilities():
    x = _rand((1, 64, 4096), 1.0, 1) + 3.0
    assert torch.equal(_run(x, 0.0, _state(1, 1)), x)
    assert torch.equal(_run(x, 2.0 ** -18, _state(1, 1)), x)                  # rounds to 0
    y = _run(x, 65535 / 65536, _state(1, 1))
    assert 0 <= int((y != 0).sum()) <= 40                                    # 4 of 262144 are to be expected
    for p in (0.1, 0.37):
        share = float((_run(x, p, _state(3, 4)) == 0).double().mean())
        assert abs(share - p) < 6 * (p * (1 - p) / x.numel()) ** 0.5 + 2.0 ** -17
        mean = float(_run(torch.ones_like(x), p, _state(3, 5)).double().mean())
        assert abs(mean - 1.0) < 6 * (p / (1 - p) / x.numel()) ** 0.5


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c,ld,shift", [(64, 72, 0), (64, 72, 8), (64, 71, 3), (40, 48, 1), (7, 9, 1), (1, 2, 1), (1024, 1032, 0)])
def test_strides_and_alignment(c, ld, shift, typ):
    """The mask goes by the element's number, not by its place: the same values, the gaps untouched."""
    n, rows = 2, 70
    x, r = _rand((n, rows, ld), 1.0, 1, typ)[..., shift:shift + c], _rand((n, rows, ld + 8), 1.0, 2, typ)[..., shift:shift + c]
    out = torch.full((n, rows, ld + 16), 9.0, device=DEV, dtype=TYPE[typ])
    for res in (None, r):
        _run(x, 0.3, _state(5, 6), 7, res, out[..., shift:shift + c])
        assert torch.equal(out[..., shift:shift + c], _run(x.contiguous(), 0.3, _state(5, 6), 7, res.contiguous() if res is not None else None))
        assert bool((torch.cat([out[..., :shift], out[..., shift + c:]], -1) == 9.0).all())


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", [256, 257])
def test_in_place(c, typ):
    x, r = _rand((2, 33, c), 1.0, 1, typ), _rand((2, 33, c), 1.0, 2, typ)
    want = _run(x, 0.2, _state(1, 2), 0, r)
    for k in range(2):
        args = [x.clone(), r.clone()]
        _run(args[0], 0.2, _state(1, 2), 0, args[1], args[k])
        assert torch.equal(args[k], want)


def test_dropped_places_may_hold_anything():
    x = _rand((1, 8, 1024), 1.0, 1)
    keep, _ = kept(0, x.numel(), 0.5, 9, 9, 9)
    dirty = x.clone()
    dirty.view(-1)[torch.from_numpy(~keep).to(DEV)] = float("nan")
    assert torch.equal(_run(dirty, 0.5, _state(9, 9), 9), _run(x, 0.5, _state(9, 9), 9))


def test_seeds_steps_and_sites_draw_anew():
    x = torch.ones((1, 64, 1024), device=DEV)
    base = _run(x, 0.5, _state(1, 1), 1) != 0
    for seed, step, site in ((2, 1, 1), (1, 2, 1), (1, 1, 2), (1 + 2 ** 32, 1, 1)):
        other = _run(x, 0.5, _state(seed, step), site) != 0
        assert abs(float((base == other).double().mean()) - 0.5) < 6 * 0.5 / x.numel() ** 0.5
    assert torch.equal(base, _run(x, 0.5, _state(1, 1 + 2 ** 32), 1) != 0)   # the step's low 32 bits count


def test_backward_is_the_same_call():
    """Differences of sum(dy y): linear in x, so they are exact to rounding."""
    x, dy = _rand((1, 4, 100), 1.0, 1), _rand((1, 4, 100), 1.0, 2)
    dx = _run(dy, 0.25, _state(3, 4), 5)
    for at in ((0, 0, 0), (0, 3, 99), (0, 2, 50)):
        ends = []
        for sign in (0.5, -0.5):
            moved = x.clone()
            moved[at] += sign
            ends.append(float((to64(_run(moved, 0.25, _state(3, 4), 5)) * to64(dy)).sum()))
        assert abs(ends[0] - ends[1] - float(dx[at])) <= 1e-4


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_offsets_beyond_32_bits(typ):
    """More than 2^32 elements' worth of counter: the last ones follow the documented numbers."""
    n, rows, c = 2, 537_000, 4000 if typ == "bf16" else 2000
    x = torch.ones((n, rows, c), device=DEV, dtype=TYPE[typ])
    y = _run(x, 0.5, _state(7, 8), 9, y=x)
    count = 80_000
    keep, scale = kept(y.numel() - count, count, 0.5, 7, 8, 9)
    assert np.array_equal(to64(y.view(-1)[-count:]), np.where(keep, scale, 0.0))


def test_captured_calls_follow_the_state():
    x, state = _rand((2, 40, 512), 1.0, 1), _state(3, 1)
    y = torch.empty_like(x)
    _run(x, 0.1, state, 2, y=y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _run(x, 0.1, state, 2, y=y)
        state[1] += 1
    for step in range(1, 4):
        graph.replay()
        assert torch.equal(y, _run(x, 0.1, _state(3, step), 2))
