"""Layer norm and its gradient against double precision.

Tolerances, with u = 2^-24: a row's sums have at most 32 serial additions a thread and 10 joining steps, so a mean is off
by at most 44 u of the mean magnitude; statistics, products and the final additions add a handful of roundings.  64 u of the
sum of the magnitudes that enter an element covers them.  The weight's gradient adds, per CTA and then over CTAs, at most
64 rows one after another at these sizes: 80 u of the sum of magnitudes.  A bf16 result adds half a unit in its last place (8 significant bits)."""
import numpy as np
import pytest
import torch

from helpers import half_unit, to64

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rand(shape, std, seed, typ="f32", mean=0.0):
    return torch.empty(shape, device=DEV).normal_(mean, std, generator=_gen(seed)).to(TYPE[typ])


def _forward(x, w, b, y=None, eps=EPS):
    from paper_2104_11981_b200 import binding as B
    n, rows, c = x.shape
    y = torch.full_like(x, float("nan")) if y is None else y
    mean, rstd = torch.full((n, rows), float("nan"), device=DEV), torch.full((n, rows), float("nan"), device=DEV)
    B.layer_norm(x, w, b, eps, y, mean, rstd)
    return y, mean, rstd


def _backward(x, dy, w, mean, rstd, bias=True, gtype="f32", dx=None):
    from paper_2104_11981_b200 import binding as B
    n, rows, c = x.shape
    dx = torch.full_like(x, float("nan")) if dx is None else dx
    g = torch.full((n, 2 * c + 3), 7.0, device=DEV, dtype=TYPE[gtype])       # the stacked gradient of the node
    dw, db = g[:, 1:c + 1], g[:, c + 2:2 * c + 2] if bias else None
    work = torch.empty(B.layer_norm_grad_workspace_bytes(n, rows, c), dtype=torch.uint8, device=DEV)
    B.layer_norm_grad(x, dy, w, mean, rstd, dx, dw, db, work)
    torch.cuda.synchronize()
    assert bool((g[:, 0] == 7.0).all()) and bool((g[:, c + 1] == 7.0).all()) and bool((g[:, 2 * c + 2] == 7.0).all())
    assert bias or bool((g[:, c + 2:] == 7.0).all())
    return dx, dw, db


def _check_forward(x, w, b, typ):
    y, mean, rstd = _forward(x, w, b)
    X, W = to64(x), to64(w)[:, None]
    Bv = to64(b)[:, None] if b is not None else 0.0
    mu = X.mean(-1, keepdims=True)
    rs = 1.0 / np.sqrt(((X - mu) ** 2).mean(-1, keepdims=True) + EPS)
    size = np.abs(X).mean(-1, keepdims=True)
    assert np.all(np.abs(to64(mean)[..., None] - mu) <= 44 * U * size + 1e-45)
    # the centred squares inherit the mean's error: relative to the deviation it is size * rs
    assert np.all(np.abs(to64(rstd)[..., None] / rs - 1) <= 64 * U * (1 + size * rs))
    want = (X - mu) * rs * W + Bv
    tol = 64 * U * ((np.abs(X) + size) * rs * np.abs(W) * (1 + np.abs((X - mu) * rs)) + np.abs(Bv)) + half_unit(typ, want)
    assert np.all(np.abs(to64(y) - want) <= tol)
    return y, mean, rstd


def _check_backward(x, dy, w, mean, rstd, typ, bias=True, gtype="f32"):
    dx, dw, db = _backward(x, dy, w, mean, rstd, bias, gtype)
    X, G, W = to64(x), to64(dy), to64(w)[:, None]
    mu, rs = to64(mean)[..., None], to64(rstd)[..., None]
    xh = (X - mu) * rs
    xsize = (np.abs(X) + np.abs(mu)) * rs                                   # what rounding in x - mu scales with
    v = G * W
    want = rs * (v - v.mean(-1, keepdims=True) - xh * (v * xh).mean(-1, keepdims=True))
    tol = 64 * U * rs * (np.abs(v) + np.abs(v).mean(-1, keepdims=True) + xsize * (np.abs(v) * xsize).mean(-1, keepdims=True)) \
        + half_unit(typ, want) + 1e-45
    assert np.all(np.abs(to64(dx) - want) <= tol)
    dwo = (G * xh).sum(1)
    assert np.all(np.abs(to64(dw) - dwo) <= 80 * U * (np.abs(G) * xsize).sum(1) + half_unit(gtype, dwo) + 1e-45)
    if bias:
        dbo = G.sum(1)
        assert np.all(np.abs(to64(db) - dbo) <= 80 * U * np.abs(G).sum(1) + half_unit(gtype, dbo) + 1e-45)
    again = _backward(x, dy, w, mean, rstd, bias, gtype)
    assert all(p is None or torch.equal(p, q) for p, q in zip((dx, dw, db), again))     # bitwise repeatable


# widths on both sides of every variant's limit: a warp's registers, a CTA's, rows read again; odd ones take single elements
WIDTHS = [1, 2, 7, 8, 64, 127, 128, 129, 256, 264, 500, 512, 513, 768, 1000, 1024, 1032, 2047, 2048, 4096, 4104, 5000, 8192, 8193,
          9001, 10_240, 12_288, 13_799, 13_900, 16_383, 16_384, 16_385,
          16_392, 32_768, 32_769, 40_000]


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", WIDTHS)
def test_widths(c, typ):
    n, rows = 2, 5 if c > 64 else 37
    x = _rand((n, rows, c), 1.5, c, typ, mean=0.3)
    w, b = _rand((n, c), 0.5, c + 1, mean=1.0), _rand((n, c), 0.3, c + 2)
    y, mean, rstd = _check_forward(x, w, b, typ)
    _check_backward(x, _rand((n, rows, c), 1e-2, c + 3, typ), w, mean, rstd, typ)


@pytest.mark.parametrize("n,rows", [(1, 1), (1, 2), (5, 1), (1, 1000), (16, 33), (300, 2), (3, 257)])
@pytest.mark.parametrize("c,typ,gtype", [(384, "bf16", "bf16"), (96, "f32", "f32"), (1536, "bf16", "f32"), (77, "f32", "bf16")])
def test_rows_and_nodes(n, rows, c, typ, gtype):
    """From one row to more rows than CTAs; weights and biases as column ranges of the stacked parameters."""
    params = _rand((n, 3 * c + 5), 1.0, 9)
    w, b = params[:, 1:c + 1], params[:, c + 4:2 * c + 4]
    x = _rand((n, rows, c), 2.0, 10, typ)
    _, mean, rstd = _check_forward(x, w, b, typ)
    _check_forward(x, w, None, typ)
    dy = _rand((n, rows, c), 1.0, 11, typ)
    _check_backward(x, dy, w, mean, rstd, typ, True, gtype)
    _check_backward(x, dy, w, mean, rstd, typ, False, gtype)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c,ld,shift", [(256, 300, 0), (256, 304, 8), (256, 304, 3), (2048, 2049, 1), (1024, 1024 + 64, 0)])
def test_strides_and_alignment(c, ld, shift, typ):
    """Rows inside wider ones, starting anywhere: the same values, the gaps untouched."""
    n, rows = 2, 6
    buf = _rand((n, rows, ld), 1.0, 5, typ)
    if shift + c > ld:
        pytest.skip("row does not fit")
    x = buf[..., shift:shift + c]
    w, b = _rand((n, c), 1.0, 6), _rand((n, c), 1.0, 7)
    out = torch.full((n, rows, ld), 9.0, device=DEV, dtype=TYPE[typ])
    y, mean, rstd = _forward(x, w, b, out[..., shift:shift + c])
    plain, pm, pr = _check_forward(x.contiguous(), w, b, typ)
    assert np.allclose(to64(y), to64(plain), rtol=2.0 ** -7 if typ == "bf16" else 1e-5, atol=1e-5)
    edge = torch.cat([out[..., :shift], out[..., shift + c:]], -1)
    assert bool((edge == 9.0).all())
    _check_backward(x, _rand((n, rows, ld), 1.0, 8, typ)[..., shift:shift + c], w, mean, rstd, typ)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", [512, 4096, 129, 40_000])
def test_in_place(c, typ):
    n, rows = 2, 19
    x, dy = _rand((n, rows, c), 1.0, 1, typ), _rand((n, rows, c), 1.0, 2, typ)
    w, b = _rand((n, c), 1.0, 3), _rand((n, c), 1.0, 4)
    y, mean, rstd = _forward(x, w, b)
    dx, dw, db = _backward(x, dy, w, mean, rstd)
    inplace = x.clone()
    _forward(inplace, w, b, inplace)
    assert torch.equal(inplace, y)
    g = dy.clone()
    r = _backward(x, g, w, mean, rstd, dx=g)
    assert torch.equal(g, dx) and torch.equal(r[1], dw) and torch.equal(r[2], db)
    g = x.clone()
    r = _backward(g, dy, w, mean, rstd, dx=g)
    assert torch.equal(g, dx) and torch.equal(r[1], dw) and torch.equal(r[2], db)


def test_calls_from_several_threads():
    """Different widths of one kernel from two host threads, each on its own stream."""
    import threading
    from paper_2104_11981_b200 import binding as B
    faults = []

    def work(c, seed):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                x, w, b = _rand((2, 40, c), 1.0, seed), _rand((2, c), 1.0, seed + 1), _rand((2, c), 1.0, seed + 2)
                first = None
                for _ in range(30):
                    y, mean, rstd = _forward(x, w, b)
                    dx, dw, db = _backward(x, y, w, mean, rstd)
                    first = first or (y, dx, dw, db)
                    stream.synchronize()
                    assert all(torch.equal(p, q) for p, q in zip(first, (y, dx, dw, db)))
        except BaseException as e:  # noqa: BLE001
            faults.append(e)

    threads = [threading.Thread(target=work, args=(c, c)) for c in (4097, 8191, 9000, 16_384)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not faults and B.kernel_error() == 0


def test_no_rows():
    x = torch.empty((3, 0, 40), device=DEV)
    w = _rand((3, 40), 1.0, 3)
    y, mean, rstd = _forward(x, w, None)
    _, dw, db = _backward(x, x.clone(), w, mean, rstd)
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_constant_and_nonfinite_rows():
    """A constant row has no deviation (y = b, finite rstd); a NaN or infinity stays within its row."""
    c = 640
    x = _rand((1, 4, c), 1.0, 3)
    x[0, 0] = 3.25
    x[0, 1, 17] = float("nan")
    x[0, 2, 600] = float("inf")
    w, b = _rand((1, c), 1.0, 4), _rand((1, c), 1.0, 5)
    y, mean, rstd = _forward(x, w, b)
    assert np.allclose(to64(y)[0, 0], to64(b)[0], atol=1e-4) and abs(float(rstd[0, 0]) - EPS ** -0.5) < 1e-3 * EPS ** -0.5
    assert torch.isnan(y[0, 1]).all() and torch.isnan(y[0, 2]).all()
    _check_forward(x[:, 3:].contiguous(), w, b, "f32")
    assert torch.isfinite(y[0, 3]).all()


def test_large_mean_small_spread():
    """The centred second sweep keeps the variance of a row whose mean is 1000 times its deviation."""
    x = _rand((2, 8, 3000), 1.0, 6, mean=1000.0)
    _check_forward(x, _rand((2, 3000), 1.0, 7), None, "f32")


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_offsets_beyond_32_bits(typ):
    """More than 2^31 elements in one array: the last rows are those of a short call on them."""
    c, rows = 4096, 532_000
    x = torch.empty((1, rows, c), device=DEV, dtype=TYPE[typ])
    x[:, -64:] = _rand((1, 64, c), 1.0, 8, typ)
    x[:, :-64] = 0.5
    w, b = _rand((1, c), 1.0, 9), _rand((1, c), 1.0, 10)
    assert x.numel() > 2 ** 31
    y, mean, rstd = _forward(x, w, b)
    ys, ms, rs = _forward(x[:, -64:].contiguous(), w, b)
    assert torch.equal(y[:, -64:], ys) and torch.equal(mean[:, -64:], ms) and torch.equal(rstd[:, -64:], rs)
    dy = torch.zeros_like(x)
    dy[:, -64:] = _rand((1, 64, c), 1.0, 11, typ)
    dx, dw, db = _backward(x, dy, w, mean, rstd, dx=y)
    sx, sw, sb = _backward(x[:, -64:].contiguous(), dy[:, -64:].contiguous(), w, ms, rs)
    assert torch.equal(dx[:, -64:], sx)
    # other rows have dy = 0: the sums differ in order only
    tol = 80 * U * np.abs(to64(dy[:, -64:])).sum(1) * 8
    assert np.all(np.abs(to64(dw) - to64(sw)) <= tol) and np.all(np.abs(to64(db) - to64(sb)) <= tol)


def test_gradient_is_the_slope_of_the_forward_pass():
    """Central differences of sum(dy y) in x, w and b.  The step 2^-6 leaves a curvature error of about step^2 and a
    rounding error of about u |y| / step: 2e-3 of the gradient's size covers both."""
    n, rows, c = 2, 3, 48
    x, dy = _rand((n, rows, c), 1.0, 1), _rand((n, rows, c), 1.0, 2)
    w, b = _rand((n, c), 0.5, 3, mean=1.0), _rand((n, c), 0.5, 4)
    _, mean, rstd = _forward(x, w, b)
    dx, dw, db = _backward(x, dy, w, mean, rstd)

    def objective(x, w, b):
        return float((to64(_forward(x, w, b)[0]) * to64(dy)).sum())

    h = 2.0 ** -6
    for what, grad, at in ((0, dx, [(0, 0, 0), (1, 2, 47), (0, 1, 20)]), (1, dw, [(0, 5), (1, 47)]), (2, db, [(1, 0), (0, 31)])):
        scale = float(to64(grad).std())
        for idx in at:
            ends = []
            for sign in (1.0, -1.0):
                args = [x.clone(), w.clone(), b.clone()]
                args[what][idx] += sign * h
                ends.append(objective(*args))
            assert abs((ends[0] - ends[1]) / (2 * h) - float(grad[idx])) <= 2e-3 * max(scale, abs(float(grad[idx])))
