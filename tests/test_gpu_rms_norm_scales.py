"""Scales of the root-mean-square norm's 8-bit output in rows that have none: zeros, NaN and infinities, squares beyond fp32."""
import pytest
import torch

from test_gpu_rms_norm import _forward, _rand

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")

# groups of eight lanes to one warp; CTAs of rows that start on 16 bytes, alike, and (apart) differently; rows read twice from memory
WIDTHS = [1, 5, 40, 100, 256, 300, 512, 640, 641, 2048, 2049, 9000, 9001, 20_000]


def _rows(c, typ, eps, apart):
    x = _rand((2, 9, c), 1.0, c, typ)
    w = _rand((2, c), 0.1, c + 1, mean=1.0)
    w[:, c // 2] = 0.0
    x[:, 1] = 0.0
    x[:, 2, c - 1] = NAN
    x[:, 3, 0] = INF
    x[:, 4, c // 2] = -INF                       # where the weight is 0
    x[:, 5] = 1e25                               # finite; its squares are not
    x[:, 6] = NAN
    x[:, 7, c // 2], x[:, 7, c - 1] = INF, NAN
    if apart:                                    # the input's rows begin elsewhere than the others'
        room = torch.empty((2, 9, c + 3), device=x.device, dtype=x.dtype)
        room[..., 1:c + 1] = x
        x = room[..., 1:c + 1]
    return x, w, _forward(x, w, eight=True, eps=eps)


@pytest.mark.parametrize("eps", [0.0, 1e-5])
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", WIDTHS)
def test_rows_without_a_scale(c, typ, apart, eps):
    _, _, (_, _, rstd, q, scales) = _rows(c, typ, eps, apart)
    assert torch.equal(scales[:, 1], torch.zeros_like(scales[:, 1])) and bool((q[:, 1].float() == 0).all())
    assert bool(torch.isnan(scales[:, [2, 3, 4, 6, 7]]).all())
    assert bool((rstd[:, [3, 4, 5]] == 0).all()) and bool((scales[:, 5] == 0).all())
    if c > 1:                                    # with one column, its weight is 0
        assert bool((scales[:, [0, 8]] > 0).all()) and bool(torch.isfinite(scales[:, [0, 8]]).all())


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", WIDTHS)
def test_other_rows_are_as_without_them(c, typ):
    """Rows beside those above, in one warp with them where rows are short, are what they are beside ordinary ones.  (At the same places: where a
    row starts within 16 bytes decides which thread adds which of its squares.)"""
    x, w, (y, h, rstd, q, scales) = _rows(c, typ, 1e-5, False)
    x[:, 1:8] = _rand((2, 7, c), 1.0, c + 2, typ)
    beside = _forward(x, w, eight=True)
    for got, want in zip((y, h, rstd, q.view(torch.uint8), scales), (*beside[:3], beside[3].view(torch.uint8), beside[4])):
        assert torch.equal(got[:, [0, 8]], want[:, [0, 8]])
