"""Clipped policy loss with a KL term, and its gradient, against double precision.

Tolerances, with u = 2^-24: the sum of exponentials has terms good to 2^-22 (the exponential) and to 2^-24 times their
exponent's size, of which those that matter are below 32, and serial additions of positive terms; 1e-5 covers a vocabulary
of 200,000.  So logp is good to 1e-5 + u |logp|, and what is formed from it by exp() to a relative 2e-5; a bf16
gradient adds half a unit in its last place (8 significant bits)."""
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


def _case(n, rows, v, typ, seed, spread=2.0, kl=True):
    gen = _gen(seed)
    s = dict(z=torch.empty((n, rows, v), device=DEV).normal_(0.0, spread, generator=gen).to(TYPE[typ]))
    s["tok"] = torch.randint(0, v, (n, rows), device=DEV, generator=gen)
    lp = torch.from_numpy(_logp64(s["z"], s["tok"])).to(DEV)
    moved = torch.empty((n, rows), device=DEV).normal_(0.0, 0.3, generator=gen)
    r = torch.exp(-moved)                                                 # keep the ratio off the objective's corners
    moved += 0.02 * (((r - 0.8).abs() < 2e-3) | ((r - 1.28).abs() < 2e-3))
    s["old"] = (lp + moved).float()
    s["ref"] = (lp + torch.empty((n, rows), device=DEV).normal_(0.0, 0.4, generator=gen)).float() if kl else None
    s["adv"] = torch.empty((n, rows), device=DEV).normal_(0.0, 1.0, generator=gen)
    s["w"] = (torch.rand((n, rows), device=DEV, generator=gen) < 0.75).float() / max(1, rows)
    s["kl"] = 0.07 if kl else 0.0
    return s


def _logp64(z, tok):
    z = to64(z)
    m = z.max(-1)
    lse = m + np.log(np.exp(z - m[..., None]).sum(-1))
    return np.take_along_axis(z, tok.cpu().numpy().clip(0, z.shape[-1] - 1)[..., None], -1)[..., 0] - lse


def _call(s, grad=True, out=None, z=None, lo=0.2, hi=0.28):
    from paper_2104_11981_b200 import binding as B
    z = s["z"] if z is None else z
    n, rows, v = z.shape
    loss, logp = torch.full((n,), float("nan"), device=DEV), torch.full((n, rows), float("nan"), device=DEV)
    d = (torch.full_like(z, float("nan")) if out is None else out) if grad else None
    work = torch.empty(B.policy_loss_workspace_bytes(n, rows, v), dtype=torch.uint8, device=DEV)
    B.policy_loss_grad(z, s["tok"], s["w"], s["adv"], s["old"], s["ref"], lo, hi, s["kl"], loss, logp, d, work)
    torch.cuda.synchronize()
    return loss, logp, d


def _truth(s, lo=0.2, hi=0.28):
    """(loss, logp, dlogits, sizes) in double; masked rows as the header states."""
    z, tok, w = to64(s["z"]), s["tok"].cpu().numpy(), to64(s["w"])
    lo, hi, kl = float(np.float32(lo)), float(np.float32(hi)), float(np.float32(s["kl"]))
    kept = (w != 0) & (tok >= 0) & (tok < z.shape[-1])
    z = np.where(kept[..., None], z, 0.0)
    with np.errstate(all="ignore"):
        m = z.max(-1, keepdims=True)
        p = np.exp(z - m)
        lse = m[..., 0] + np.log(p.sum(-1))
        p /= p.sum(-1, keepdims=True)
    safe = np.where(kept, tok, 0)
    lp = np.where(kept, np.take_along_axis(z, safe[..., None], -1)[..., 0] - lse, 0.0)
    adv, old = to64(s["adv"]), to64(s["old"])
    r = np.exp(lp - old)
    a, b = r * adv, np.clip(r, 1 - lo, 1 + hi) * adv
    term, slope, size = -np.minimum(a, b), np.where(a <= b, -a, 0.0), np.abs(a)
    if s["ref"] is not None:
        far = to64(s["ref"]) - lp
        term, slope = term + kl * (np.exp(far) - far - 1), slope + kl * (1 - np.exp(far))
        size = size + kl * (1 + np.exp(far) + np.abs(far))
    w = np.where(kept, w, 0.0)
    onehot = np.zeros_like(z)
    np.put_along_axis(onehot, safe[..., None], 1.0, -1)
    d = (w * slope)[..., None] * (onehot - p)
    return (w * term).sum(1), lp, d, dict(loss=(np.abs(w) * size).sum(1), d=(np.abs(w) * size)[..., None] * (onehot + p))


def _check(s, typ, got):
    loss, logp, d = got
    lo, lpo, do, size = _truth(s)
    assert np.all(np.abs(to64(logp) - lpo) <= 1e-5 + U * np.abs(lpo))
    assert np.all(np.abs(to64(loss) - lo) <= 4e-5 * size["loss"] + U * np.abs(lo))
    if d is not None:
        # tiny probabilities may flush to zero
        assert np.all(np.abs(to64(d) - do) <= 4e-5 * size["d"] + half_unit(typ, do) + 1e-38)


VOCABS = [1, 2, 7, 8, 9, 63, 255, 512, 1000, 4095, 4096, 4097, 8191, 32_768, 50_001, 65_536, 100_003, 131_072, 200_000]


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("v", VOCABS)
def test_vocabularies(v, typ):
    for n, rows, kl in ((2, 9, True), (1, 1, False)):
        s = _case(n, rows, v, typ, v + rows, kl=kl)
        first = _call(s)
        _check(s, typ, first)
        again = _call(s)
        assert all(torch.equal(p, q) for p, q in zip(first, again))                # bitwise repeatable
        only = _call(s, grad=False)
        assert torch.equal(only[0], first[0]) and torch.equal(only[1], first[1])
        z = s["z"].clone()
        inplace = _call(s, out=z, z=z)
        assert all(torch.equal(p, q) for p, q in zip(first, inplace))


@pytest.mark.parametrize("n,rows", [(1, 1), (1, 3), (7, 1), (3, 50), (2, 700), (150, 2)])
def test_rows_and_nodes(n, rows):
    for typ, v in (("bf16", 3000), ("f32", 1111)):
        s = _case(n, rows, v, typ, n + rows)
        _check(s, typ, _call(s))


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("v,ldz,ldd,shift", [(1000, 1001, 1001, 0), (1000, 1008, 1016, 8), (1000, 1003, 1003, 3), (999, 1024, 999, 0),
                                              (40_000, 40_001, 40_003, 1)])
def test_strides_and_alignment(v, ldz, ldd, shift, typ):
    s = _case(2, 5, v, typ, 3)
    buf = torch.full((2, 5, ldz), float("nan"), device=DEV, dtype=TYPE[typ])
    shift = min(shift, ldz - v)
    z = buf[..., shift:shift + v]
    z.copy_(s["z"])
    out = torch.full((2, 5, ldd), 9.0, device=DEV, dtype=TYPE[typ])
    got = _call(s, out=out[..., :v], z=z)
    _check(s, typ, got)
    assert bool((out[..., v:] == 9.0).all())


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("v", [777, 40_000])
def test_masked_rows(v, typ):
    """Weight 0 or a token outside the vocabulary: nothing of the row shows, whatever its logits are; a node without a
    single kept row has loss 0 and no gradient."""
    s = _case(3, 8, v, typ, 5)
    s["w"][:] = 0.125
    s["w"][0, 1] = 0.0
    s["z"][0, 1] = float("nan")
    s["tok"][0, 2], s["tok"][0, 3], s["tok"][0, 4] = -100, v, 2 ** 40
    s["z"][0, 2] = float("inf")
    s["z"][0, 3] = -float("inf")
    s["old"][0, 3] = float("nan")
    s["w"][1] = 0.0
    s["z"][1] = float("nan")
    s["ref"][1] = float("inf")
    s["w"][2, 0] = -0.5                                                    # a weight may have either sign
    got = _call(s)
    clean = {k: (t.clone() if torch.is_tensor(t) else t) for k, t in s.items()}
    for k in ("old", "ref", "adv"):
        clean[k] = torch.where(torch.isfinite(clean[k]), clean[k], 0.0)
    _check(clean, typ, got)
    assert float(got[0][1]) == 0.0 and bool((got[2][1] == 0).all()) and bool((got[1][1] == 0).all())
    assert bool((got[2][0, 1:5] == 0).all())


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_forbidden_tokens_and_large_logits(typ):
    """Logits of minus infinity or of the type's lowest value have probability 0 and gradient 0; a shift of every logit by
    a large constant, or one dominating logit, changes no more than its rounding does."""
    v = 5000
    s = _case(1, 6, v, typ, 6)
    keep = torch.zeros(v, dtype=torch.bool, device=DEV)
    keep[::3] = True
    keep[s["tok"].flatten()] = True
    s["z"][0, 0, ~keep] = -float("inf")
    s["z"][0, 1, ~keep] = torch.finfo(TYPE[typ]).min
    s["z"][0, 2] = -float("inf")
    s["z"][0, 2, s["tok"][0, 2]] = 1.0                                      # certainty
    s["z"][0, 3] *= 20.0
    s["z"][0, 4] += 256.0
    s["z"][0, 5, :4000] = -float("inf")                                     # whole threads see nothing
    s["tok"][0, 5] = 4500
    lp = torch.from_numpy(_logp64(s["z"], s["tok"])).to(DEV)
    s["old"], s["ref"] = (lp + 0.1).float(), (lp - 0.2).float()
    s["w"][:] = 1.0
    got = _call(s)
    # rows 3 and 4: the exponent's rounding is u |z| log2(e), |z| up to 300: 300 * 1.45 * 2^-24 = 2.6e-5 more
    loss, logp, d = got
    lo, lpo, do, size = _truth(s)
    assert np.all(np.abs(to64(logp) - lpo) <= 4e-5 + U * np.abs(lpo))
    assert np.all(np.abs(to64(d) - do) <= 1.5e-4 * size["d"] + half_unit(typ, do) + 1e-38)
    assert bool((d[0, 0, ~keep] == 0).all()) and bool((d[0, 1, ~keep] == 0).all())
    assert -1e-5 <= float(logp[0, 2]) <= 0.0


def test_corners_of_the_objective():
    """Both signs of the advantage on both sides of the interval, inside it, and A = 0."""
    v, rows = 64, 10
    s = _case(1, rows, v, "f32", 9)
    lp = torch.from_numpy(_logp64(s["z"], s["tok"])).to(DEV)[0]
    ratios = torch.tensor([0.5, 0.5, 1.0, 1.0, 2.0, 2.0, 0.81, 1.27, 0.5, 2.0], device=DEV)
    s["old"][0] = (lp - torch.log(ratios)).float()
    s["adv"][0] = torch.tensor([1.0, -1.0, 1.0, -1.0, 1.0, -1.0, -1.0, 1.0, 0.0, 0.0], device=DEV)
    s["w"][:] = 1.0
    s["ref"], s["kl"] = None, 0.0
    got = _call(s)
    _check(s, "f32", got)
    flat = (got[2][0].abs().sum(-1) == 0).cpu().tolist()
    assert flat == [False, True, False, False, True, False, False, False, True, True]   # held back, or nothing to gain


def test_gradient_is_the_slope_of_the_loss():
    """Central differences of the loss in single logits, step 2^-5: curvature error about step^2, rounding about
    u |loss| / step; 3e-3 of the largest slope covers both."""
    n, rows, v = 1, 4, 40
    s = _case(n, rows, v, "f32", 21, spread=1.0)
    lp = torch.from_numpy(_logp64(s["z"], s["tok"])).to(DEV)
    s["old"] = (lp + 0.05).float()                                         # away from the corners for the whole step
    s["w"][:] = 1.0
    d = _call(s)[2]
    h, top = 2.0 ** -5, float(d.abs().max())
    for r in range(rows):
        for k in (int(s["tok"][0, r]), 0, 39):
            ends = []
            for sign in (1.0, -1.0):
                z = s["z"].clone()
                z[0, r, k] += sign * h
                ends.append(float(_call(s, grad=False, z=z)[0][0]))
            assert abs((ends[0] - ends[1]) / (2 * h) - float(d[0, r, k])) <= 3e-3 * max(top, 1.0)


def test_offsets_beyond_32_bits():
    """More than 2^31 logits: the last rows are those of a short call on them."""
    v, rows = 131_072, 16_400
    assert v * rows > 2 ** 31
    s = _case(1, 8, v, "bf16", 2)
    z = torch.zeros((1, rows, v), device=DEV, dtype=torch.bfloat16)
    z[:, -8:] = s["z"]
    big = dict(z=z, kl=s["kl"])
    for k in ("tok", "old", "ref", "adv", "w"):
        big[k] = torch.zeros((1, rows), device=DEV, dtype=s[k].dtype)
        big[k][:, -8:] = s[k]
    short, long = _call(s), _call(big, out=z, z=z)                          # in place: the gradient over the logits
    assert torch.equal(long[1][:, -8:], short[1]) and torch.equal(z[:, -8:], short[2])
    assert abs(float(long[0][0]) - float(short[0][0])) <= 2 * U * abs(float(short[0][0]))
    assert bool((z[:, :-8].view(torch.int16) == 0).all())


def test_streams_and_graphs():
    s = _case(2, 30, 5000, "bf16", 4)
    from paper_2104_11981_b200 import binding as B
    eager = _call(s)
    loss, logp, d = torch.empty(2, device=DEV), torch.empty((2, 30), device=DEV), torch.empty_like(s["z"])
    work = torch.empty(B.policy_loss_workspace_bytes(2, 30, 5000), dtype=torch.uint8, device=DEV)
    args = (s["z"], s["tok"], s["w"], s["adv"], s["old"], s["ref"], 0.2, 0.28, s["kl"], loss, logp, d, work)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.policy_loss_grad(*args, stream=side)
    side.synchronize()
    assert torch.equal(d, eager[2]) and torch.equal(loss, eager[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.policy_loss_grad(*args)
    d.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(d, eager[2]) and torch.equal(loss, eager[0]) and torch.equal(logp, eager[1])
