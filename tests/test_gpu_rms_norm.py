"""Root-mean-square norm with residual, its 8-bit output and its gradient against double precision.

Tolerances, with u = 2^-24.  h = x + residual is one addition: u |h|, and what is stored of it half a unit of its type.  A sum of squares
has no cancellation; a thread adds at most 40 of them one after another and 10 joining steps follow, so it is off by at most 50 u of
itself, rstd by half of that and two units for the root: 32 u covers it and the rounding of h.  y adds two products: 40 u |y|.  The gradient adds
a row's products v xh the same way: 64 u of the sum of their magnitudes, and the weight's gradient, at these sizes, at most 64 rows one after
another per CTA and then over CTAs: 80 u.  In 8 bits q is off the unrounded quotient by half a step of e4m3, 2^-4 of the value or 2^-10 below
2^-6, after at most eight fp32 roundings."""
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


def _forward(x, w, r=None, h=None, y=None, eight=False, keep=True, only8=False, eps=EPS):
    from paper_2104_11981_b200 import binding as B
    n, rows, c = x.shape
    h = torch.full_like(x, float("nan")) if keep and h is None else h
    y = None if only8 else torch.full_like(x, float("nan")) if y is None else y
    rstd = torch.full((n, rows), float("nan"), device=DEV)
    q = torch.full((n, rows, c), 1, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn) if eight else None
    scales = torch.full((n, rows), float("nan"), device=DEV) if eight else None
    B.rms_norm(x, w, eps, y, rstd, r, h, q, scales)
    return y, h, rstd, q, scales


def _check_forward(x, w, r, typ, eight=False, only8=False):
    y, h, rstd, q, scales = _forward(x, w, r, eight=eight, only8=only8)
    H = to64(x) + (to64(r) if r is not None else 0.0)
    rs = 1.0 / np.sqrt((H ** 2).mean(-1, keepdims=True) + EPS)
    assert np.all(np.abs(to64(h) - H) <= U * np.abs(H) + half_unit(typ, H) * (1 + 2.0 ** -14) + 1e-45)
    assert np.all(np.abs(to64(rstd)[..., None] / rs - 1) <= 32 * U)
    want = H * rs * to64(w)[:, None]
    if not only8:
        assert np.all(np.abs(to64(y) - want) <= 40 * U * np.abs(want) + half_unit(typ, want) * (1 + 2.0 ** -14) + 1e-45)
    if eight:
        top = np.abs(want).max(-1, keepdims=True)
        assert np.all(np.abs(to64(scales)[..., None] - top / 448) <= 40 * U * top / 448)
        v = np.divide(want * 448, top, out=np.zeros_like(want), where=top > 0)
        got = to64(q.float())
        assert np.isfinite(got).all() and np.abs(got).max() <= 448
        assert np.all(np.abs(got - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10) + 8 * U * 448)
    return y, h, rstd


def _backward(h, dy, w, rstd, dres=None, gtype="f32", dh=None):
    from paper_2104_11981_b200 import binding as B
    n, rows, c = h.shape
    dh = torch.full_like(h, float("nan")) if dh is None else dh
    g = torch.full((n, c + 3), 7.0, device=DEV, dtype=TYPE[gtype])            # the stacked gradient of the node
    dw = g[:, 1:c + 1]
    work = torch.full((B.rms_norm_grad_workspace_bytes(n, rows, c),), 255, dtype=torch.uint8, device=DEV)
    B.rms_norm_grad(h, dy, w, rstd, dh, dw, work, dres)
    torch.cuda.synchronize()
    assert bool((g[:, 0] == 7.0).all()) and bool((g[:, c + 1:] == 7.0).all())
    return dh, dw


def _check_backward(h, dy, w, rstd, typ, dres=None, gtype="f32"):
    dh, dw = _backward(h, dy, w, rstd, dres, gtype)
    H, G, W, rs = to64(h), to64(dy), to64(w)[:, None], to64(rstd)[..., None]
    E = to64(dres) if dres is not None else np.zeros_like(H)
    xh, v = H * rs, G * W
    want = E + rs * (v - xh * (v * xh).mean(-1, keepdims=True))
    tol = 64 * U * (np.abs(E) + rs * (np.abs(v) + np.abs(xh) * np.abs(v * xh).mean(-1, keepdims=True))) + half_unit(typ, want) * (1 + 2.0 ** -10) + 1e-45
    assert np.all(np.abs(to64(dh) - want) <= tol)
    dwo = (G * xh).sum(1)
    assert np.all(np.abs(to64(dw) - dwo) <= 80 * U * np.abs(G * xh).sum(1) + half_unit(gtype, dwo) * (1 + 2.0 ** -10) + 1e-45)
    again = _backward(h, dy, w, rstd, dres, gtype)
    assert torch.equal(dh, again[0]) and torch.equal(dw, again[1])          # bitwise repeatable


# widths on both sides of every variant's limit: a warp's registers, a CTA's, rows read again; odd ones take single elements
WIDTHS = [1, 2, 7, 8, 64, 127, 128, 129, 256, 264, 500, 512, 513, 768, 1000, 1024, 1032, 2047, 2048, 4096, 4104, 5000, 8192, 8193,
          9001, 10_240, 12_288, 13_799, 13_900, 16_383, 16_384, 16_385, 16_392, 32_769, 40_000]


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", WIDTHS)
def test_widths(c, typ):
    n, rows = 2, 5 if c > 64 else 37
    x, r = _rand((n, rows, c), 1.5, c, typ, mean=0.3), _rand((n, rows, c), 2.0, c + 4, typ)
    w = _rand((n, c), 0.5, c + 1, mean=1.0)
    y, h, rstd = _check_forward(x, w, r, typ)
    _check_forward(x, w, None, typ)
    dy = _rand((n, rows, c), 1e-2, c + 3, typ)
    _check_backward(h, dy, w, rstd, typ, _rand((n, rows, c), 1e-2, c + 5, typ))
    _check_backward(h, dy, w, rstd, typ)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", WIDTHS)
def test_eight_bits(c, typ):
    n, rows = 2, 3 if c > 64 else 19
    x, r, w = _rand((n, rows, c), 1.0, c, typ), _rand((n, rows, c), 1.0, c + 1, typ), _rand((n, c), 0.5, c + 2, mean=1.0)
    x[0, 1], r[0, 1] = 0.0, 0.0                                              # a row of zeros
    _check_forward(x, w, r, typ, eight=True)
    _check_forward(x, w, None, typ, eight=True, only8=True)
    both, alone = _forward(x, w, r, eight=True), _forward(x, w, r, eight=True, only8=True, keep=False)
    assert torch.equal(both[3].view(torch.uint8), alone[3].view(torch.uint8)) and torch.equal(both[4], alone[4])
    assert torch.equal(both[0], _forward(x, w, r)[0])                        # and the wide output is that of a call without them


@pytest.mark.parametrize("n,rows", [(1, 1), (1, 2), (5, 1), (1, 1000), (16, 33), (300, 2), (3, 257)])
@pytest.mark.parametrize("c,typ,gtype", [(384, "bf16", "bf16"), (96, "f32", "f32"), (1536, "bf16", "f32"), (77, "f32", "bf16")])
def test_rows_and_nodes(n, rows, c, typ, gtype):
    """From one row to more rows than CTAs; weights as column ranges of the stacked parameters."""
    params = _rand((n, 3 * c + 5), 1.0, 9)
    w = params[:, 1:c + 1]
    x, r = _rand((n, rows, c), 2.0, 10, typ), _rand((n, rows, c), 1.0, 12, typ)
    _, h, rstd = _check_forward(x, w, r, typ)
    _check_backward(h, _rand((n, rows, c), 1.0, 11, typ), w, rstd, typ, r, gtype)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c,ld,shift", [(256, 300, 0), (256, 304, 8), (256, 304, 3), (2048, 2049, 1), (1024, 1024 + 64, 0), (40, 41, 1)])
def test_strides_and_alignment(c, ld, shift, typ):
    """Rows inside wider ones, starting anywhere, each array with a stride of its own: the same values, the gaps untouched."""
    n, rows = 2, 6
    x, r, dy = (_rand((n, rows, ld + k), 1.0, 5 + k, typ)[..., shift:shift + c] for k in range(3))
    w = _rand((n, c), 1.0, 8)
    out = [torch.full((n, rows, ld + 8), 9.0, device=DEV, dtype=TYPE[typ]) for _ in range(3)]
    h, y, dh = (o[..., shift:shift + c] for o in out)
    _, _, rstd, _, _ = _forward(x, w, r, h, y)
    _backward(h, dy, w, rstd, r, dh=dh)
    plain_y, plain_h, plain_rstd = _check_forward(x.contiguous(), w, r.contiguous(), typ)
    plain_dh, _ = _backward(plain_h, dy.contiguous(), w, plain_rstd, r.contiguous())
    for got, want in ((y, plain_y), (h, plain_h), (dh, plain_dh)):
        assert np.allclose(to64(got), to64(want), rtol=2.0 ** -7 if typ == "bf16" else 1e-5, atol=1e-5)
    for o in out:
        assert bool((torch.cat([o[..., :shift], o[..., shift + c:]], -1) == 9.0).all())
    _check_backward(h, dy, w, rstd, typ, r)
    q = torch.full((n, rows, ld + 8), 77, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn)
    from paper_2104_11981_b200 import binding as B
    scales = torch.empty((n, rows), device=DEV)
    B.rms_norm(x, w, EPS, None, rstd, r, None, q[..., shift:shift + c], scales)
    want = _forward(x.contiguous(), w, r.contiguous(), eight=True)
    assert torch.equal(q.view(torch.uint8)[..., shift:shift + c], want[3].view(torch.uint8))
    assert bool((torch.cat([q.view(torch.uint8)[..., :shift], q.view(torch.uint8)[..., shift + c:]], -1) == 77).all())


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", [512, 4096, 129, 12_288, 40_000])
def test_in_place(c, typ):
    n, rows = 2, 19
    x, r, dy = (_rand((n, rows, c), 1.0, k, typ) for k in range(3))
    w = _rand((n, c), 1.0, 3)
    y, h, rstd, _, _ = _forward(x, w, r)
    for hp, yp in ((0, 1), (1, 0)):                                          # h over x and y over the residual, and the other way about
        places = [x.clone(), r.clone()]
        _forward(places[0], w, places[1], h=places[hp], y=places[yp])
        assert torch.equal(places[hp], h) and torch.equal(places[yp], y)
    dh, dw = _backward(h, dy, w, rstd, r)
    for k in range(3):
        args = [h.clone(), dy.clone(), r.clone()]
        got = _backward(args[0], args[1], w, rstd, args[2], dh=args[k])
        assert torch.equal(args[k], dh) and torch.equal(got[1], dw)


def test_no_rows():
    x = torch.empty((3, 0, 40), device=DEV)
    w = _rand((3, 40), 1.0, 3)
    _forward(x, w, x, eight=True)
    _, dw = _backward(x, x, w, torch.empty((3, 0), device=DEV))
    assert bool((dw == 0).all())


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", [640, 641, 20_000])
def test_nonfinite_and_extreme_rows(c, typ):
    """A NaN or infinity stays within its row (its scale is NaN); tiny and large rows keep their 8-bit digits."""
    x = _rand((1, 6, c), 1.0, 3, typ)
    x[0, 1, 17] = float("nan")
    x[0, 2, 600] = float("inf")
    x[0, 3] = (x[0, 3].double() * 2.0 ** -120).to(x.dtype)
    x[0, 4] = (x[0, 4].double() * 2.0 ** 50).to(x.dtype)
    w = _rand((1, c), 0.1, 4, mean=1.0)
    y, h, rstd, q, scales = _forward(x, w, eight=True)
    assert torch.isnan(y[0, 1]).all() and torch.isnan(scales[0, 1:3]).all() and float(rstd[0, 2]) == 0.0
    ok = [0, 3, 4, 5]
    assert torch.isfinite(y[0, ok].float()).all() and torch.isfinite(scales[0, ok]).all()
    v = to64(x)[0, ok] * to64(w)[0]
    v = v * 448 / np.abs(v).max(-1, keepdims=True)
    assert np.all(np.abs(to64(q.float())[0, ok] - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10) + 8 * U * 448)
    _check_forward(x[:, [0, 4, 5]].contiguous(), w, None, typ, eight=True)


def test_zero_row_without_eps_is_nan_and_stays_alone():
    x = _rand((1, 3, 256), 1.0, 3)
    x[0, 1] = 0.0
    y, _, rstd, _, _ = _forward(x, _rand((1, 256), 1.0, 4), eps=0.0)
    assert torch.isnan(y[0, 1]).all() and torch.isinf(rstd[0, 1]) and torch.isfinite(y[0, ::2]).all()


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_offsets_beyond_32_bits(typ):
    """More than 2^31 elements in one array: the last rows are those of a short call on them."""
    c, rows = 4096, 532_000
    x = torch.empty((1, rows, c), device=DEV, dtype=TYPE[typ])
    x[:, -64:] = _rand((1, 64, c), 1.0, 8, typ)
    x[:, :-64] = 0.5
    w = _rand((1, c), 1.0, 9)
    assert x.numel() > 2 ** 31
    y, _, rstd, _, _ = _forward(x, w, keep=False)
    ys, _, rs, _, _ = _forward(x[:, -64:].contiguous(), w, keep=False)
    assert torch.equal(y[:, -64:], ys) and torch.equal(rstd[:, -64:], rs)
    dy = torch.zeros_like(x)
    dy[:, -64:] = _rand((1, 64, c), 1.0, 11, typ)
    dh, dw = _backward(x, dy, w, rstd, dh=y)
    sh, sw = _backward(x[:, -64:].contiguous(), dy[:, -64:].contiguous(), w, rs)
    assert torch.equal(dh[:, -64:], sh)
    # other rows have dy = 0: the sums differ in order only
    assert np.all(np.abs(to64(dw) - to64(sw)) <= 80 * U * np.abs(to64(dy[:, -64:])).sum(1) * 8)


def test_gradient_is_the_slope_of_the_forward_pass():
    """Central differences of sum(dy y) + sum(dres h) in x, the residual and w.  The step 2^-6 leaves a curvature error of about step^2 and a
    rounding error of about u |y| / step: 2e-3 of the gradient's size covers both."""
    n, rows, c = 2, 3, 48
    x, r, dy, dres = (_rand((n, rows, c), 1.0, k) for k in range(4))
    w = _rand((n, c), 0.5, 5, mean=1.0)
    _, h, rstd, _, _ = _forward(x, w, r)
    dh, dw = _backward(h, dy, w, rstd, dres)

    def objective(x, r, w):
        y, h, _, _, _ = _forward(x, w, r)
        return float((to64(y) * to64(dy)).sum() + (to64(h) * to64(dres)).sum())

    step = 2.0 ** -6
    for what, grad, at in ((0, dh, [(0, 0, 0), (1, 2, 47)]), (1, dh, [(0, 1, 20), (1, 0, 3)]), (2, dw, [(0, 5), (1, 47)])):
        for idx in at:
            ends = []
            for sign in (1.0, -1.0):
                args = [x.clone(), r.clone(), w.clone()]
                args[what][idx] += sign * step
                ends.append(objective(*args))
            assert abs((ends[0] - ends[1]) / (2 * step) - float(grad[idx])) <= 2e-3 * max(float(to64(grad).std()), abs(float(grad[idx])))


def test_calls_from_several_threads():
    """Different widths of one kernel from host threads, each on its own stream."""
    import threading
    from paper_2104_11981_b200 import binding as B
    faults = []

    def work(c):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                x, r, w = _rand((2, 40, c), 1.0, c), _rand((2, 40, c), 1.0, c + 2), _rand((2, c), 1.0, c + 1)
                first = None
                for _ in range(30):
                    y, h, rstd, q, _ = _forward(x, w, r, eight=True)
                    dh, dw = _backward(h, y, w, rstd, x)
                    first = first or (y, h, dh, dw)
                    stream.synchronize()
                    assert all(torch.equal(p, q) for p, q in zip(first, (y, h, dh, dw)))
        except BaseException as e:  # noqa: BLE001
            faults.append(e)

    threads = [threading.Thread(target=work, args=(c,)) for c in (4097, 8184, 9000, 16_384)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not faults and B.kernel_error() == 0


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("n,rows", [(1, 1), (1, 2), (2, 1), (2, 9), (3, 700)])
@pytest.mark.parametrize("c", [9, 61, 777, 2100, 5001, 9000])
def test_rows_that_start_alike(c, n, rows, typ):
    """All arrays begin at the same odd place and have the same odd stride: rows in chunks whose ends belong to others.  The first and the
    last row begin and end where the memory of the array does."""
    if n * rows > 100 and c > 3000:
        rows = 50
    ld, shift = c + 3, 1 if typ == "bf16" else 3
    count = (n * rows - 1) * ld + c                                           # nothing behind the last row
    def place(seed, std=1.0):
        flat = _rand((count + shift,), std, seed, typ)
        return flat, torch.as_strided(flat, (n, rows, c), (rows * ld, ld, 1), shift)
    (_, x), (_, r), (_, dy) = (place(k) for k in range(3))
    (fh, h), (fy, y), (fd, dh) = (place(k) for k in range(3, 6))
    before = [f.clone() for f in (fh, fy, fd)]
    w = _rand((n, c), 0.5, 8, mean=1.0)
    _, _, rstd, _, _ = _forward(x, w, r, h, y)
    _backward(h, dy, w, rstd, r, dh=dh)
    _check_forward(x, w, r, typ)
    _check_backward(h, dy, w, rstd, typ, r)
    py, ph, prstd, q, scales = _forward(x.contiguous(), w, r.contiguous(), eight=True)
    assert torch.equal(h, ph)
    assert np.allclose(to64(y), to64(py), rtol=2.0 ** -7 if typ == "bf16" else 1e-5, atol=1e-5)
    gaps = torch.ones(count + shift, dtype=torch.bool, device=DEV)
    torch.as_strided(gaps, (n, rows, c), (rows * ld, ld, 1), shift).fill_(False)
    for now, was in zip((fh, fy, fd), before):
        assert torch.equal(now[gaps], was[gaps])
    from paper_2104_11981_b200 import binding as B
    q8 = torch.full((n, rows, c), 9, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn)
    B.rms_norm(x, w, EPS, None, rstd, r, None, q8, scales)
    assert torch.equal(q8.view(torch.uint8), q.view(torch.uint8))
