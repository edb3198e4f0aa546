"""The two ways by which the binding reads tensors (their exchange interface, or their attributes) make the same calls and refuse the same
tensors; other devices, streams and views."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(params=["interface", "attributes"])
def binding(request, monkeypatch):
    from paper_2104_11981_b200 import binding as B
    B._home()
    if request.param == "interface":
        assert B._direct is not None, "the tensors' exchange interface is expected here"
    else:
        monkeypatch.setattr(B, "_direct", None)
    return B


def _r(*shape, seed=0, typ=torch.float32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 1)
    return torch.empty(shape, device=DEV).normal_(0.0, 1.0, generator=g).to(typ)


def test_calls(binding):
    B, bf16 = binding, torch.bfloat16
    n, rows, c, vocab = 2, 3, 40, 70
    params = _r(n, vocab * c + c + 5)
    table, weight = params[:, 2:2 + vocab * c].unflatten(1, (vocab, c)), params[:, 3 + vocab * c:3 + (vocab + 1) * c]
    tokens = torch.tensor([[1, 69, -1], [70, 0, 5]], device=DEV)
    y = torch.empty((n, rows, c), device=DEV, dtype=bf16)
    B.embedding(table, tokens, y, 2.0)
    want = torch.zeros((n, rows, c), device=DEV)
    for i, r, t in ((0, 0, 1), (0, 1, 69), (1, 1, 0), (1, 2, 5)):
        want[i, r] = 2 * table[i, t]
    assert torch.equal(y, want.to(bf16))
    g = torch.full_like(params, 7.0)
    work = torch.empty(B.embedding_grad_workspace_bytes(n, rows, vocab, c), dtype=torch.uint8, device=DEV)
    dt = g[:, 2:2 + vocab * c].unflatten(1, (vocab, c))
    B.embedding_grad(tokens, y, dt, work, 0.5)
    assert torch.equal(dt[0, 69], y[0, 1].float() * 0.5) and int((dt != 0).any(-1).sum()) == 4 and bool((g[:, :2] == 7).all())
    B.embedding_grad(tokens, y, dt, work, 0.5, accumulate=True)
    assert torch.equal(dt[1, 5], y[1, 2].float())
    x, res = _r(n, rows, c, seed=3, typ=bf16), _r(n, rows, c + 8, seed=4, typ=bf16)[..., 8:]
    h, q = torch.empty_like(x), torch.empty((n, rows, c), device=DEV, dtype=torch.float8_e4m3fn)
    rstd, scales = torch.empty((n, rows), device=DEV), torch.empty((n, rows), device=DEV)
    B.rms_norm(x, weight, 1e-5, y, rstd, res, h, q, scales)
    H = x.double() + res.double()
    want = H * (H.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * weight.double()[:, None]
    assert float((y.double() - want).norm() / want.norm()) < 4e-3 and torch.equal(h, H.to(bf16))
    assert float((q.double() * scales.double()[..., None] - want).norm() / want.norm()) < 0.06
    only = torch.empty_like(rstd)
    B.rms_norm(x, weight, 1e-5, None, only, res, None, q, scales)
    B.rms_norm(x, weight, 1e-5, y, only)
    dh, dw = torch.empty_like(x), torch.full((n, c + 1), 5.0, device=DEV, dtype=bf16)
    work = torch.empty(B.rms_norm_grad_workspace_bytes(n, rows, c), dtype=torch.uint8, device=DEV)
    B.rms_norm_grad(h, y, weight, rstd, dh, dw[:, 1:], work, res)
    xh = h.double() * rstd.double()[..., None]
    assert float((dw[:, 1:].double() - (y.double() * xh).sum(1)).abs().max()) < 0.1 and bool((dw[:, 0] == 5).all())
    B.dropout(x, 0.5, torch.tensor([1, 2], device=DEV), y, 3, res)
    assert 0.3 < float((y == res).double().mean()) < 0.7
    z = _r(n, rows, vocab)
    allowed = torch.full((n, rows, 3), -1, dtype=torch.int32, device=DEV)
    allowed[0, 0, 0] = ~1
    one = torch.full((n, rows), 2.0, device=DEV)
    start = torch.tensor([0, 2, 2, 2, 2, 2, 3], device=DEV)
    out = torch.empty_like(z)
    B.logits_adjust(z, out, params[:, :vocab], allowed, torch.tensor([5, 5, 9], device=DEV), start, one, one, one, one)
    w = (z + params[:, None, :vocab]) / 2
    w[0, 0, 5] = ((z[0, 0, 5] / 2 if z[0, 0, 5] > 0 else z[0, 0, 5] * 2) - 6 + params[0, 5]) / 2
    w[1, 2, 9] = ((z[1, 2, 9] / 2 if z[1, 2, 9] > 0 else z[1, 2, 9] * 2) - 4 + params[1, 9]) / 2
    w[0, 0, 0] = -float("inf")
    assert torch.allclose(out, w, rtol=1e-5, atol=1e-6)
    B.logits_adjust_grad(z, out, z, allowed[:1, :1].expand(n, rows, 3), torch.tensor([5, 5, 9], device=DEV), start, one, one)
    assert bool((out[..., 0] == 0).all()) and torch.allclose(out[1, 0, 1:], z[1, 0, 1:] / 2)
    B.logits_adjust_grad(z, out)
    assert torch.equal(out, z)


def test_refusals(binding):
    B = binding
    x, w, r = _r(2, 3, 40), _r(2, 40), torch.empty((2, 3), device=DEV)
    y, state = torch.empty_like(x), torch.zeros(2, dtype=torch.int64, device=DEV)
    bad = (AssertionError, TypeError, AttributeError, ValueError, B.DecentlamError)
    for args in ((x.double(), w, 1e-5, y, r), (x, w.bfloat16(), 1e-5, y, r), (x, w, 1e-5, y[:, :2], r), (x, w, 1e-5, y.bfloat16(), r),
                 (x, w, 1e-5, y, r[:, :2]), (x, w[:, :39], 1e-5, y, r), (x.cpu(), w, 1e-5, y, r), (x, w.cpu(), 1e-5, y, r),
                 (x, w, 1e-5, y, r.double()), (x, w, 1e-5, y, r, x.bfloat16()), (x, w, 1e-5, y, r, None, None, y.bfloat16(), r),
                 (x.permute(0, 2, 1), w, 1e-5, y, r), (x[0], w, 1e-5, y, r), (None, w, 1e-5, y, r), (x, None, 1e-5, y, r), ("x", w, 1e-5, y, r)):
        with pytest.raises(bad):
            B.rms_norm(*args)
    with pytest.raises(B.DecentlamError):
        B.rms_norm(x, w, -1.0, y, r)
    for args in ((x, 0.1, state[:1], y), (x, 0.1, state.int(), y), (x, 0.1, state.cpu(), y), (x, "p", state, y), (x, 0.1, state, y.half())):
        with pytest.raises(bad):
            B.dropout(*args)
    with pytest.raises(B.DecentlamError):
        B.dropout(x, 1.0, state, y)
    tokens = torch.zeros((2, 3), dtype=torch.int64, device=DEV)
    table = _r(2, 5, 40)
    for args in ((table.permute(0, 2, 1), tokens, y), (table[:, ::2], tokens, y), (table, tokens.int(), y), (table, tokens[:, :2], y),
                 (table, tokens, y[..., :39]), (table.half(), tokens, y)):
        with pytest.raises(bad):
            B.embedding(*args)
    one, text, start = torch.ones((2, 3), device=DEV), tokens.view(-1), torch.zeros(7, dtype=torch.int64, device=DEV)
    for kw in (dict(allowed=torch.zeros((2, 3, 1), dtype=torch.int32, device=DEV)), dict(allowed=torch.zeros((2, 3, 2), device=DEV)),
               dict(history=text), dict(history=text, history_start=start[:6]), dict(history=text.int(), history_start=start),
               dict(temperature=one[:, :2]), dict(bias=_r(2, 39)), dict(bias=_r(2, 40).half())):
        with pytest.raises(bad):
            B.logits_adjust(x, y, **kw)
    with pytest.raises(B.DecentlamError):
        B.logits_adjust(x, y, repetition=one)                                # a penalty without texts
    work = torch.empty(64, dtype=torch.uint8, device=DEV)
    for w2 in (work, work.cpu()):
        with pytest.raises(bad):
            B.embedding_grad(tokens, x, table, w2)
    torch.cuda.synchronize()


def test_streams(binding):
    B = binding
    x, y = _r(4, 500, 512), torch.empty((4, 500, 512), device=DEV)
    state = torch.tensor([1, 1], device=DEV)
    B.dropout(x, 0.5, state, y)
    want = y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for k in range(2):
        y.zero_()
        side.wait_stream(torch.cuda.current_stream())
        if k == 0:
            B.dropout(x, 0.5, state, y, stream=side)
        else:
            with torch.cuda.stream(side):
                B.dropout(x, 0.5, state, y)
        side.synchronize()
        assert torch.equal(y, want)


def test_tensors_that_learn(binding):
    """Parameters and views of them, as a training program holds them."""
    B = binding
    x = torch.nn.Parameter(_r(2, 3, 40))
    y = torch.empty((2, 3, 40), device=DEV)
    with torch.no_grad():
        B.dropout(x, 0.0, torch.zeros(2, dtype=torch.int64, device=DEV), y)
    assert np.array_equal(y.cpu().numpy(), x.detach().cpu().numpy())
