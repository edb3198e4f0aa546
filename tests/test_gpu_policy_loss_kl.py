"""The KL term of the policy loss while the policy is still close to its reference, against double precision."""
import numpy as np
import pytest
import torch

from helpers import to64
from test_gpu_policy_loss import DEV, U, _call, _gen
from test_gpu_policy_loss_range import _scores

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("v", [64, 1111])
@pytest.mark.parametrize("rows", [50, 640])
def test_kl_term_near_its_zero(rows, v):
    """Advantage 0 leaves the KL term alone: q = e^u - u - 1 and its slope 1 - e^u, u = ref - logp from 1e-4 to 3 in size, taken
    from the logp that the call returns, so that its rounding does not enter.  u is exact to 2^-24.  For |u| < 1/2 everything formed
    from it is good to a few roundings: 8 u q.  Beyond, the exponential is good to 2^-22 and its exponent is rounded: 8 u (1 + |u|) e^u.
    The weight and kl add two roundings each.  The gradient row is slope (onehot - p), p good to a relative 1e-5 and logp's 2^-24 |logp|."""
    z = torch.empty((1, rows, v), device=DEV).normal_(0.0, 1.0, generator=_gen(v))
    tok = torch.randint(0, v, (1, rows), device=DEV, generator=_gen(v + 1))
    s = _scores(z, tok, 3, kl=1.0)
    s["adv"].zero_()
    logp = _call(s, grad=False)[1]
    far = torch.from_numpy(np.resize(np.array([1e-4, -1e-4, 1e-3, -1e-3, 3e-3, -5e-3, 1e-2, -1e-2, 0.1, -0.1, 0.49, -0.49, 0.51,
                                               -0.51, 1.5, -3.0, 0.0]), rows)).to(DEV)[None]
    s["ref"] = (logp.double() + far).float()
    s["ref"][far == 0] = logp[far == 0]
    u, w = to64(s["ref"]) - to64(logp), to64(s["w"])
    q = np.expm1(u) - u
    small = np.abs(u) < 0.4
    q[small] = (u ** 2 * (0.5 + u * (1 / 6 + u * (1 / 24 + u * (1 / 120 + u * (1 / 720 + u * (1 / 5040 + u * (1 / 40320 + u * (
        1 / 362880 + u * (1 / 3628800 + u / 39916800))))))))))[small]
    err = np.where(np.abs(u) < 0.5, 8 * U * q, 8 * U * (1 + np.abs(u)) * np.exp(u))
    one = np.zeros((1, rows), bool)
    for r in range(min(rows, 17)):                                        # each row by itself, then all of them
        one[:] = False
        one[0, r] = True
        alone = dict(s, w=torch.where(torch.from_numpy(one).to(DEV), s["w"], 0.0))
        assert abs(float(_call(alone, grad=False)[0][0]) - (w * q)[0, r]) <= (w * (err + 4 * U * q))[0, r] + 1e-45
    loss, again, d = _call(s)
    assert torch.equal(again, logp)
    assert abs(float(loss[0]) - (w * q).sum()) <= (w * (err + 4 * U * q)).sum() + U * (w * q).sum()
    p = np.exp(to64(z) - to64(z).max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    hot = np.zeros_like(p)
    np.put_along_axis(hot, tok.cpu().numpy()[..., None], 1.0, -1)
    slope = (w * -np.expm1(u))[..., None]
    assert np.all(np.abs(to64(d) - slope * (hot - p)) <= 2e-5 * np.abs(slope) * (hot + p) + 1e-38)
    assert bool((d[far == 0] == 0).all())
