"""Embedding and its gradient against double precision.

Tolerances, with u = 2^-24: the forward pass is one product and one rounding.  The sum of a row's k gradients in any order is off by at most
k u of the sum of their magnitudes; scale, the addition to what was there and the joining of blocks are four more roundings."""
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


def _tokens(n, rows, vocab, seed, kind="uniform"):
    if kind == "one":
        return torch.full((n, rows), vocab - 1, device=DEV)
    if kind == "text":                                                        # few common tokens, many rare ones
        u = torch.rand((n, rows), device=DEV, generator=_gen(seed), dtype=torch.float64)
        return (torch.exp(u * np.log(vocab + 1)) - 1).long().clamp(0, vocab - 1)
    t = torch.randint(0, vocab, (n, rows), device=DEV, generator=_gen(seed))
    if kind == "stray":                                                       # a third of them stand for none
        t[:, ::3] = torch.tensor([-1, vocab, 2 ** 40, -2 ** 63, vocab + 1], device=DEV).repeat(rows)[:t[:, ::3].shape[1]]
    return t


def _forward(table, tokens, typ, scale=1.0, y=None):
    from paper_2104_11981_b200 import binding as B
    y = torch.full((*tokens.shape, table.shape[2]), float("nan"), device=DEV, dtype=TYPE[typ]) if y is None else y
    B.embedding(table, tokens, y, scale)
    return y


def _check_forward(table, tokens, typ, scale):
    y = _forward(table, tokens, typ, scale)
    T, k, vocab = to64(table), tokens.cpu().numpy(), table.shape[1]
    ok = (k >= 0) & (k < vocab)
    want = np.stack([T[i][np.where(ok[i], k[i], 0)] * ok[i][:, None] for i in range(T.shape[0])]) * float(np.float32(scale))
    assert np.all(np.abs(to64(y) - want) <= U * np.abs(want) + half_unit(typ, want) * (1 + 2.0 ** -14))
    if scale == 1.0 and typ == "f32":
        assert np.array_equal(to64(y), want)


def _backward(tokens, dy, vocab, gtype, scale=1.0, add=None, pad=0, work=None):
    """add: what the gradient holds before; pad: further columns of the stacked gradient on both sides."""
    from paper_2104_11981_b200 import binding as B
    n, rows, c = dy.shape
    g = torch.full((n, vocab * c + 2 * pad), 7.0, device=DEV, dtype=TYPE[gtype])
    dt = g[:, pad:pad + vocab * c].view(n, vocab, c) if pad == 0 else torch.as_strided(g, (n, vocab, c), (g.stride(0), c, 1), pad)
    if add is not None:
        dt.copy_(add)
    if work is None:
        work = torch.full((B.embedding_grad_workspace_bytes(n, rows, vocab, c),), 255, dtype=torch.uint8, device=DEV)
    B.embedding_grad(tokens, dy, dt, work, scale, accumulate=add is not None)
    assert pad == 0 or (bool((g[:, :pad] == 7.0).all()) and bool((g[:, -pad:] == 7.0).all()))
    return dt


def _check_backward(tokens, dy, vocab, gtype, scale=1.0, add=None, pad=0):
    got = _backward(tokens, dy, vocab, gtype, scale, add, pad)
    n, rows, c = dy.shape
    G, k, s = to64(dy), tokens.cpu().numpy(), float(np.float32(scale))
    for i in range(n):
        ok = (k[i] >= 0) & (k[i] < vocab)
        want, size = np.zeros((vocab, c)), np.zeros((vocab, c))
        np.add.at(want, k[i][ok], G[i][ok] * s)
        np.add.at(size, k[i][ok], np.abs(G[i][ok] * s))
        count = np.bincount(k[i][ok], minlength=vocab)[:, None]
        if add is not None:
            want += to64(add[i])
            size += np.abs(to64(add[i]))
        out = to64(got[i])
        assert np.all(np.abs(out - want) <= (count + 4) * U * size + half_unit(gtype, want) * (1 + 2.0 ** -10))
        if add is None:
            assert np.all(out[count[:, 0] == 0] == 0)
        else:
            assert np.array_equal(out[count[:, 0] == 0], to64(add[i])[count[:, 0] == 0])     # left as they were
    assert torch.equal(got, _backward(tokens, dy, vocab, gtype, scale, add, pad))             # bitwise repeatable


@pytest.mark.parametrize("typ,ttype", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,rows,vocab,c", [(1, 1, 1, 1), (1, 1, 5000, 4096), (3, 65, 77, 8), (2, 1000, 500, 129), (4, 33, 64, 768),
                                            (2, 7, 100, 1032), (1, 5, 9, 20_000), (300, 2, 10, 40)])
def test_forward(n, rows, vocab, c, typ, ttype):
    table = _rand((n, vocab, c), 1.0, c, ttype)
    _check_forward(table, _tokens(n, rows, vocab, 1), typ, 1.0)
    _check_forward(table, _tokens(n, rows, vocab, 2, "stray"), typ, 11.3)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 4, 8])
def test_forward_from_columns_of_the_stacked_parameters(shift, typ):
    n, vocab, c, rows = 3, 50, 64, 21
    params = _rand((n, vocab * c + 37), 1.0, 3)
    table = torch.as_strided(params, (n, vocab, c), (params.stride(0), c, 1), shift)
    tokens = _tokens(n, rows, vocab, 4)
    out = torch.full((n, rows, c + 24), 9.0, device=DEV, dtype=TYPE[typ])
    _forward(table, tokens, typ, 2.0, out[..., shift:shift + c])
    assert torch.equal(out[..., shift:shift + c], _forward(table.contiguous(), tokens, typ, 2.0))
    assert bool((torch.cat([out[..., :shift], out[..., shift + c:]], -1) == 9.0).all())


SHAPES = [(1, 1, 1, 1), (1, 1, 300, 4096), (3, 65, 77, 8), (2, 300, 500, 129), (4, 63, 64, 768), (1, 64, 65, 1032), (2, 2048, 40, 33),
          (2, 2049, 1000, 40), (1, 5000, 131_073, 24), (1, 16_384, 700, 64), (2, 16_385, 300, 65), (1, 70_000, 2000, 16), (300, 3, 10, 40)]


@pytest.mark.parametrize("typ,gtype", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("kind", ["text", "stray", "one"])
@pytest.mark.parametrize("n,rows,vocab,c", SHAPES)
def test_gradient(n, rows, vocab, c, kind, typ, gtype):
    tokens = _tokens(n, rows, vocab, rows, kind)
    dy = _rand((n, rows, c), 1.0, c, typ)
    _check_backward(tokens, dy, vocab, gtype, 1.0 if kind == "one" else 3.7)


@pytest.mark.parametrize("gtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["text", "stray"])
@pytest.mark.parametrize("n,rows,vocab,c", [(2, 300, 500, 128), (1, 5000, 900, 65), (3, 1, 10, 8)])
def test_gradient_is_added(n, rows, vocab, c, kind, gtype):
    """To a head's gradient in a column range of the stacked gradient that starts anywhere."""
    tokens, dy = _tokens(n, rows, vocab, 5, kind), _rand((n, rows, c), 1.0, 6, "bf16")
    _check_backward(tokens, dy, vocab, gtype, 0.5, add=_rand((n, vocab, c), 1.0, 7, gtype))
    _check_backward(tokens, dy, vocab, gtype, 0.5, add=_rand((n, vocab, c), 1.0, 7, gtype), pad=3)
    _check_backward(tokens, dy, vocab, gtype, 0.5, pad=8)


def test_gradient_of_strided_rows():
    n, rows, vocab, c = 2, 200, 90, 64
    tokens = _tokens(n, rows, vocab, 5)
    wide = _rand((n, rows, c + 24), 1.0, 6, "bf16")
    for shift in (0, 8, 3):
        dy = wide[..., shift:shift + c]
        assert torch.equal(_backward(tokens, dy, vocab, "f32"), _backward(tokens, dy.contiguous(), vocab, "f32"))


def test_rows_of_strays_are_not_read():
    """What a row holds does not matter where its token stands for none."""
    tokens, dy = _tokens(2, 100, 50, 1, "stray"), _rand((2, 100, 72), 1.0, 2)
    clean = _backward(tokens, dy, 50, "f32").clone()
    dy[(tokens < 0) | (tokens >= 50)] = float("nan")
    assert torch.equal(_backward(tokens, dy, 50, "f32"), clean)


@pytest.mark.parametrize("rows", [1, 3000])
def test_no_rows_and_none_known(rows):
    empty = torch.empty((2, 0), dtype=torch.int64, device=DEV)
    assert bool((_backward(empty, torch.empty((2, 0, 24), device=DEV), 70, "bf16") == 0).all())
    add = _rand((2, 70, 24), 1.0, 1)
    assert torch.equal(_backward(empty, torch.empty((2, 0, 24), device=DEV), 70, "f32", add=add), add)
    _forward(_rand((2, 5, 24), 1.0, 1), empty, "f32")
    none = torch.full((2, rows), -7, device=DEV)
    assert bool((_backward(none, _rand((2, rows, 24), 1.0, 1), 70, "f32") == 0).all())
    assert bool((_forward(add, none, "f32") == 0).all())


def test_a_smaller_call_in_a_larger_ones_workspace():
    """What an earlier call left in the workspace does not matter."""
    from paper_2104_11981_b200 import binding as B
    work = torch.full((B.embedding_grad_workspace_bytes(2, 20_000, 900, 64),), 170, dtype=torch.uint8, device=DEV)
    calls = [(_tokens(2, rows, 900, rows, "text"), _rand((2, rows, 64), 1.0, rows)) for rows in (20_000, 300, 2500, 1)]
    for tokens, dy in calls + calls[::-1]:
        assert torch.equal(_backward(tokens, dy, 900, "f32", work=work), _backward(tokens, dy, 900, "f32"))


def test_offsets_beyond_32_bits():
    """A table of more than 2^31 elements, and its gradient."""
    n, vocab, c, rows = 2, 140_001, 8192, 40
    table = torch.empty((n, vocab, c), device=DEV, dtype=torch.bfloat16)
    for i in range(n):
        table[i].copy_(torch.arange(vocab, device=DEV)[:, None] % 251 + i)
    tokens = torch.randint(vocab - 100, vocab, (n, rows), device=DEV, generator=_gen(1))
    y = _forward(table, tokens, "bf16")
    want = (tokens % 251 + torch.arange(n, device=DEV)[:, None]).to(torch.bfloat16)[..., None]
    assert bool((y == want).all())
    from paper_2104_11981_b200 import binding as B
    work = torch.empty(B.embedding_grad_workspace_bytes(n, rows, vocab, c), dtype=torch.uint8, device=DEV)
    ones = torch.ones((n, rows, c), device=DEV, dtype=torch.bfloat16)
    B.embedding_grad(tokens, ones, table, work)                              # over the table's own memory
    for i in range(n):
        count = torch.bincount(tokens[i], minlength=vocab)
        assert all(bool((table[i, a:a + 10_000].float() == count[a:a + 10_000, None]).all()) for a in range(0, vocab, 10_000))


def test_gradient_is_the_slope_of_the_forward_pass():
    """The operator is linear: differences are exact to rounding."""
    n, rows, vocab, c = 2, 50, 9, 16
    table, tokens, dy = _rand((n, vocab, c), 1.0, 1), _tokens(n, rows, vocab, 2), _rand((n, rows, c), 1.0, 3)
    grad = _backward(tokens, dy, vocab, "f32", 1.5)
    for idx in ((0, 0, 0), (1, 8, 15), (0, 4, 7)):
        ends = []
        for sign in (0.5, -0.5):
            moved = table.clone()
            moved[idx] += sign
            ends.append(float((to64(_forward(moved, tokens, "f32", 1.5)) * to64(dy)).sum()))
        assert abs(ends[0] - ends[1] - float(grad[idx])) <= 1e-4


def test_captured_calls_see_new_tokens_and_share_a_workspace():
    """Two captured gradients with one workspace, replayed in turn on one stream, with eager calls between them."""
    from paper_2104_11981_b200 import binding as B
    n, vocab, c = 2, 600, 48
    work = torch.empty(B.embedding_grad_workspace_bytes(n, 3000, vocab, c), dtype=torch.uint8, device=DEV)
    sets = []
    for rows in (3000, 100):
        s = dict(tokens=_tokens(n, rows, vocab, rows), dy=_rand((n, rows, c), 1.0, rows), g=torch.empty((n, vocab, c), device=DEV))
        _backward(s["tokens"], s["dy"], vocab, "f32")                         # once outside capture
        s["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(s["graph"]):
            B.embedding_grad(s["tokens"], s["dy"], s["g"], work)
        sets.append(s)
    for turn in range(3):
        for s in sets:
            s["tokens"].copy_(_tokens(*s["tokens"].shape, vocab, turn, "text"))
            s["graph"].replay()
            assert torch.equal(s["g"], _backward(s["tokens"], s["dy"], vocab, "f32"))


@pytest.mark.parametrize("typ,gtype", [("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows", [2, 31, 32, 33, 64, 65, 200, 256, 511, 512, 513])
@pytest.mark.parametrize("c", [40, 1001, 1200])
def test_gradient_of_short_texts(rows, c, typ, gtype):
    """Around the sizes where a CTA has the whole text; tokens that fill several tiles, in one strip of columns and in several."""
    for vocab, kind in ((3, "uniform"), (900, "text"), (5, "stray")):
        tokens, dy = _tokens(2, rows, vocab, rows, kind), _rand((2, rows, c), 1.0, c, typ)
        _check_backward(tokens, dy, vocab, gtype, 1.5)
        _check_backward(tokens, dy, vocab, gtype, 1.5, add=_rand((2, vocab, c), 1.0, 9, gtype))


@pytest.mark.parametrize("runs", [(512,), (1, 511), (511, 1), (64,) * 8, (63, 1, 64, 200, 184), (1,) * 130 + (250,) + (1,) * 132, (100, 157), (5,) * 61])
@pytest.mark.parametrize("c", [64, 777])
def test_short_texts_whose_runs_cross_the_shares(c, runs):
    """Runs of equal tokens that begin before a share of the sorted places and end behind it; the last run stands for no token."""
    rows, vocab = sum(runs), 300
    ids = torch.repeat_interleave(torch.arange(len(runs)), torch.tensor(runs))
    ids[ids == len(runs) - 1] = vocab if len(runs) > 1 else 0
    order = torch.randperm(rows, generator=torch.Generator().manual_seed(c))
    tokens = torch.stack([ids[order], ids.flip(0)]).to(DEV)
    _check_backward(tokens, _rand((2, rows, c), 1.0, c), vocab, "f32")
