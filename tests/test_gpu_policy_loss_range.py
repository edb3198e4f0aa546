"""Policy loss over the whole range of finite logits, in every form that the kernel takes: forbidden tokens marked by any of the
usual constants, so many of them that whole threads, warps and CTAs see nothing else; rows of the mark alone; large logits.

Tolerances as in test_gpu_policy_loss: an exponent (v - m) log2(e), m the largest of the row, has two roundings of 2^-24 of
itself and log2(e)'s own 2^-26; the terms that matter are below 32, so 32 * 0.7 * 2.3 * 2^-24 = 3e-6 at their (small) end, next to
2^-22 from the exponential: 1e-5 + u |logp| covers logp, a relative 2e-5 what exp() makes of it, and a bf16 gradient adds half a
unit in its last place."""
import numpy as np
import pytest
import torch

from helpers import half_unit, to64
from test_gpu_policy_loss import DEV, TYPE, U, _call, _gen

pytestmark = pytest.mark.gpu
MARKS = [-1e4, -1e9, -1e10, -1e12, -1e18, -1e20, -1e30, -1e35, -1e37, -1e38, "lowest", -float("inf")]

# (vocabulary, rows): a warp per row, 128 and 256 threads per row, clusters, clusters that hold a part of the row
FORMS = {"bf16": [(1000, 620), (1001, 40), (12_000, 160), (40_000, 40), (300_001, 40)],
         "f32": [(900, 620), (901, 40), (6001, 160), (40_000, 40), (150_001, 40)]}
CASES = [(typ, v, rows) for typ in FORMS for v, rows in FORMS[typ]]


def _mark(k, typ):
    m = MARKS[k % len(MARKS)]
    return torch.finfo(TYPE[typ]).min if m == "lowest" else m


def _scores(z, tok, seed, kl=0.07):
    """The rest of a case whose tokens have a moderate log-probability."""
    n, rows, v = z.shape
    gen = _gen(seed)
    x = to64(z)
    m = x.max(-1, keepdims=True)
    with np.errstate(all="ignore"):
        lse = np.log(np.exp(x - m).sum(-1))
    lp = torch.from_numpy(np.take_along_axis(x - m, tok.cpu().numpy()[..., None], -1)[..., 0] - lse).to(DEV)
    assert float(lp.min()) > -60.0
    moved = torch.empty((n, rows), device=DEV).normal_(0.0, 0.3, generator=gen)
    r = torch.exp(-moved)                                                 # off the objective's corners
    moved += 0.02 * (((r - 0.8).abs() < 2e-3) | ((r - 1.28).abs() < 2e-3))
    return dict(z=z, tok=tok, old=(lp + moved).float(), ref=(lp + 0.3).float(), kl=kl,
                adv=torch.empty((n, rows), device=DEV).normal_(0.0, 1.0, generator=gen),
                w=torch.full((n, rows), 1.0 / rows, device=DEV))


def _truth(s):
    """(loss, logp, dlogits, sizes) in double, clipping to 0.8 .. 1.28.  The row's largest logit is taken off before anything else: beside
    one of 1e38 even double keeps nothing of a logarithm."""
    z, w = to64(s["z"]), to64(s["w"])
    at = s["tok"].cpu().numpy()[..., None]
    lo, hi, kl = (float(np.float32(v)) for v in (0.2, 0.28, s["kl"]))
    z = z - z.max(-1, keepdims=True)
    p = np.exp(z)
    total = p.sum(-1, keepdims=True)
    lp = np.take_along_axis(z, at, -1)[..., 0] - np.log(total[..., 0])
    kept = w != 0
    lp = np.where(kept, lp, 0.0)
    p /= total
    adv, far = to64(s["adv"]), to64(s["ref"]) - lp
    r = np.exp(lp - to64(s["old"]))
    a, b = r * adv, np.clip(r, 1 - lo, 1 + hi) * adv
    term = -np.minimum(a, b) + kl * (np.exp(far) - far - 1)
    slope = np.where(a <= b, -a, 0.0) + kl * (1 - np.exp(far))
    size = np.abs(a) + kl * (1 + np.exp(far) + np.abs(far))
    hot = np.zeros_like(z)
    np.put_along_axis(hot, at, 1.0, -1)
    return ((w * term).sum(1), lp, (w * slope)[..., None] * (hot - p),
            dict(loss=(w * size).sum(1), d=(w * size)[..., None] * (hot + p)))


def _check(s, typ):
    loss, logp, d = _call(s)
    lo, lpo, do, size = _truth(s)
    assert np.all(np.abs(to64(logp) - lpo) <= 1e-5 + U * np.abs(lpo))
    assert np.all(np.abs(to64(loss) - lo) <= 4e-5 * size["loss"] + U * np.abs(lo))
    assert np.all(np.abs(to64(d) - do) <= 4e-5 * size["d"] + half_unit(typ, do) + 1e-38)
    only = _call(s, grad=False)
    assert torch.equal(only[0], loss) and torch.equal(only[1], logp)
    return d


@pytest.mark.parametrize("typ,v,rows", CASES)
def test_every_form(typ, v, rows):
    """Ordinary logits, every third row masked by its weight: loss, log-probabilities and gradient of all forms."""
    z = torch.empty((1, rows, v), device=DEV).normal_(0.0, 2.0, generator=_gen(v)).to(TYPE[typ])
    s = _scores(z, torch.randint(0, v, (1, rows), device=DEV, generator=_gen(v + 1)), v + 2)
    s["w"][:, ::3] = 0.0
    d = _check(s, typ)
    assert bool((d[:, ::3] == 0).all()) and bool((d[:, 1].abs().sum(-1) > 0).all())


@pytest.mark.parametrize("typ,v,rows", CASES)
def test_marks_that_cover_threads_warps_and_ctas(typ, v, rows):
    """Row by row another mark, over the first half, the second half, or all but three tokens."""
    gen = _gen(v + 3)
    z = torch.empty((1, rows, v), device=DEV).normal_(0.0, 2.0, generator=gen).to(TYPE[typ])
    tok = torch.zeros((1, rows), dtype=torch.int64, device=DEV)
    forbidden = torch.zeros((1, rows, v), dtype=torch.bool, device=DEV)
    for r in range(rows):
        pattern = r // len(MARKS) % 3
        if pattern < 2:
            forbidden[0, r, :v // 2] = pattern == 0
            forbidden[0, r, v // 2:] = pattern == 1
            tok[0, r] = (3 * v // 4 if pattern == 0 else v // 4) + r % 7
        else:
            allowed = torch.tensor([r % v, v // 3 + r % 50, v - 1 - r % 9], device=DEV)
            forbidden[0, r] = True
            forbidden[0, r, allowed] = False
            tok[0, r] = allowed[r % 3]
        z[0, r, forbidden[0, r]] = _mark(r, typ)
    s = _scores(z, tok, v + 4)
    d = _check(s, typ)
    assert bool((d[forbidden] == 0).all())


@pytest.mark.parametrize("typ,v,rows", CASES)
def test_rows_of_the_mark_alone_and_large_logits(typ, v, rows):
    """A kept row that holds nothing but one finite value is uniform, whatever the value; one logit far above the others has
    all the probability; logits that differ by little at a large offset keep their differences."""
    gen = _gen(v + 5)
    z = torch.empty((1, rows, v), device=DEV).normal_(0.0, 2.0, generator=gen).to(TYPE[typ])
    tok = torch.randint(0, v, (1, rows), device=DEV, generator=gen)
    top = [1e5, 1e9, 1e10, 1e20, 1e30, 1e38, torch.finfo(TYPE[typ]).max]
    for r in range(rows):
        if r % 3 == 0:
            m = _mark(r // 3, typ)
            z[0, r] = m if np.isfinite(m) else -3e38
        elif r % 3 == 1:
            z[0, r, tok[0, r]] = top[r // 3 % len(top)]
        elif typ == "f32":
            k = torch.randint(0, 6, (v,), device=DEV, generator=gen).float()
            z[0, r] = (2.0 * k + 3e7) * (-1.0 if r % 2 else 1.0)         # a unit in the last place is 2 there
            tok[0, r] = int(z[0, r].argmax())
    _check(_scores(z, tok, v + 6), typ)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_rows_of_minus_infinity(typ):
    """No token is allowed: 0 / 0, as the formula says, in that row alone; masked by its weight it is not looked at."""
    z = torch.empty((2, 4, 3000), device=DEV).normal_(0.0, 2.0, generator=_gen(5)).to(TYPE[typ])
    tok = torch.randint(0, 3000, (2, 4), device=DEV, generator=_gen(6))
    s = _scores(z, tok, 7)
    z[0, 1] = z[1, 2] = -float("inf")
    s["w"][1, 2] = 0.0
    loss, logp, d = _call(s)
    bad = torch.zeros((2, 4), dtype=torch.bool, device=DEV)
    bad[0, 1] = True
    assert torch.equal(torch.isnan(logp), bad) and torch.equal(torch.isnan(d).all(-1), bad) and torch.equal(torch.isnan(d).any(-1), bad)
    assert bool(torch.isnan(loss[0])) and bool(torch.isfinite(loss[1]))


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_no_rows(typ):
    z = torch.empty((3, 0, 500), device=DEV, dtype=TYPE[typ])
    none = torch.empty((3, 0), device=DEV)
    s = dict(z=z, tok=none.long(), old=none, ref=none, adv=none, w=none, kl=0.1)
    loss, logp, d = _call(s)
    assert bool((loss == 0).all()) and logp.shape == (3, 0) and d.shape == z.shape
