"""Layer norm and its gradient where every group of threads takes many rows: the rows' slots in shared memory are filled again
three times over, and the weight's gradient adds up row after row, for every width class, alignment and number of rows in flight.

The reference is plain double precision (on the GPU, for its size).  Tolerances as in test_gpu_layer_norm, whose bounds do not
depend on the number of rows but for the weight's gradient: a node's rows are added in some order, which takes no sum through more
than `rows` additions, and a product has 24 roundings at the most."""
import pytest
import torch

from test_gpu_layer_norm import DEV, EPS, TYPE, U, _backward, _forward, _rand

pytestmark = pytest.mark.gpu

# a width at the top of every class, aligned and not, and the rows above 8192 columns whose number in flight differs
ALIGNED = [64, 128, 256, 512, 1024, 1536, 2048, 4096, 8192, 9216, 12_288, 16_384]
ODD = [63, 127, 255, 511, 1023, 1535, 2047, 4095, 8191, 9001, 12_001, 13_799, 16_383]


def _ctas(threads, depth, row_bytes):
    """(CTAs that an SM holds at the most, groups in each) where `threads` share a row and `depth` rows are in flight."""
    block = max(128, threads) if threads != 64 else 64
    groups = block // threads
    return max(1, min(2048 // block, (226 << 10) // (groups * depth * row_bytes))), groups


def _nodes_and_rows(c, typ):
    """So many nodes that each has two CTAs at the most, and rows for each of their groups to take more than three times as many as
    it has in flight."""
    size = (2 if typ == "bf16" else 4) * c
    ahead = next((t for top, t in ((256, 8), (512, 16), (1024, 32), (2048, 64), (4096, 128), (8192, 256)) if c <= top), 512)
    middle = 128 if typ == "bf16" else 256
    back = next((t for top, t in ((128, 8), (256, 16), (512, 32), (1024, 64), (2048, middle), (4096, 256)) if c <= top), 512)
    depth = 4 if ahead <= 64 else 3
    held = [_ctas(ahead, 4 if ahead <= 64 else 2, size), _ctas(back, 4 if back <= 64 else 3 if back < 512 else 1, 2 * size)]
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    n = min(2048, -(-sms * max(per_sm for per_sm, _ in held) // 2))
    return n, (3 * depth + 1) * 2 * max(groups for _, groups in held) + 1


def _half_unit(typ, v):
    e = torch.frexp(v)[1] - (8 if typ == "bf16" else 24)
    return torch.where(v == 0.0, torch.zeros_like(v), torch.ldexp(torch.full_like(v, 0.5), e))


def _within(got, want, tol):
    far = (got.double() - want).abs() - tol
    assert bool((far <= 0).all()), float(far.max())                       # a NaN fails too


def _check(n, rows, c, typ, seed):
    x = _rand((n, rows, c), 1.5, seed, typ, mean=0.3)
    w, b = _rand((n, c), 0.5, seed + 1, mean=1.0), _rand((n, c), 0.3, seed + 2)
    y, mean, rstd = _forward(x, w, b)
    X, W, Bv = x.double(), w.double()[:, None], b.double()[:, None]
    mu = X.mean(-1, keepdim=True)
    rs = 1.0 / torch.sqrt(((X - mu) ** 2).mean(-1, keepdim=True) + EPS)
    size = X.abs().mean(-1, keepdim=True)
    _within(mean[..., None], mu, 44 * U * size)
    _within(rstd[..., None].double() / rs, torch.ones_like(rs), 64 * U * (1 + size * rs))
    want = (X - mu) * rs
    scale = (X.abs() + size) * rs * W.abs() * (1 + want.abs()) + Bv.abs()
    want = want * W + Bv
    _within(y, want, 64 * U * scale + _half_unit(typ, want))
    del scale, want, y
    dy = _rand((n, rows, c), 1.0, seed + 3, typ)
    dx, dw, db = _backward(x, dy, w, mean, rstd)
    G, mu, rs = dy.double(), mean.double()[..., None], rstd.double()[..., None]
    xh, xsize = (X - mu) * rs, (X.abs() + mu.abs()) * rs
    _within(dw, (G * xh).sum(1), (rows + 24) * U * (G.abs() * xsize).sum(1))
    _within(db, G.sum(1), (rows + 24) * U * G.abs().sum(1))
    v = G * W
    want = rs * (v - v.mean(-1, keepdim=True) - xh * (v * xh).mean(-1, keepdim=True))
    v = v.abs()
    tol = 64 * U * rs * (v + v.mean(-1, keepdim=True) + xsize * (v * xsize).mean(-1, keepdim=True))
    _within(dx, want, tol + _half_unit(typ, want))
    del want, tol, v, G, xh, xsize, X
    again = _forward(x, w, b)
    assert torch.equal(again[1], mean) and torch.equal(again[2], rstd)
    assert all(torch.equal(p, q) for p, q in zip(_backward(x, dy, w, mean, rstd), (dx, dw, db)))    # bitwise repeatable


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", ALIGNED + ODD)
def test_many_rows_a_group(c, typ):
    n, rows = _nodes_and_rows(c, typ)
    _check(n, rows, c, typ, c)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", [16_392, 20_001])
def test_many_rows_of_the_widest(c, typ):
    """Rows that are swept from memory: one CTA a node, five rows each."""
    _check(300, 5, c, typ, c)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("c", [48, 2047, 2048, 5000])
def test_one_node_with_more_rows_than_groups(c, typ):
    """All CTAs on one node: its weight's gradient is joined from as many parts as there are."""
    _check(1, 60_000 if c < 64 else 9001, c, typ, c + 1)
