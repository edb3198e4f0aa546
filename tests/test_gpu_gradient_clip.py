"""Gradient lists: per-node norms over many tensors and clipping, against double-precision sums.

Tolerances, with u = 2^-24: a thread adds at most 36 squares in fp32 (one piece is 8192 elements over 256 threads, and
its ends), everything after that is double, so the sum is off by at most 38 u and its root by 19 u, plus one rounding:
20 u.  The scale adds three roundings, the product one; a bf16 result half a unit in its last place (8 significant bits)."""
import ctypes

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


def _nodes(n, sizes, types, seed, shift=0, std=1e-3):
    """Lists of gradients of n nodes; every tensor starts `shift` elements into its allocation."""
    gen, nodes = _gen(seed), []
    for _ in range(n):
        node = []
        for k, typ in zip(sizes, types):
            buf = torch.empty(k + shift, device=DEV).normal_(0.0, std, generator=gen).to(TYPE[typ])
            node.append(buf[shift:])
        nodes.append(node)
    return nodes


def _norm64(node):
    return np.sqrt(sum(float(np.sum(to64(t) ** 2)) for t in node))


def _check_clip(nodes, offsets, max_norm, dst, columns_extra=0):
    from paper_2104_11981_b200 import binding as B
    n = len(nodes)
    lst = B.gradients_build(nodes, offsets=offsets)
    norms = torch.full((n,), float("nan"), device=DEV)
    before = [[t.clone() for t in node] for node in nodes]
    out = torch.full((n, lst.columns + columns_extra), 7.0, device=DEV, dtype=TYPE[dst])
    B.gradient_clip(lst, max_norm, norms, out)
    torch.cuda.synchronize()
    covered = np.zeros(out.shape[1], bool)
    for i, node in enumerate(nodes):
        want = _norm64(node)
        assert abs(float(norms[i]) - want) <= 20 * U * want
        s = min(1.0, max_norm / (want + 1e-6))
        row = to64(out[i])
        for t, (g, o) in enumerate(zip(node, lst.offsets)):
            assert torch.equal(g, before[i][t])                      # gathering leaves the tensors alone
            x = to64(g) * s
            assert np.all(np.abs(row[o:o + g.numel()] - x) <= np.abs(x) * 24 * U + half_unit(dst, x) + 1e-45)
            covered[o:o + g.numel()] = True
    assert np.all(to64(out)[:, ~covered] == 7.0)                      # columns of no tensor are not touched
    first, first_norms = out.clone(), norms.clone()
    out.fill_(3.0)
    B.gradient_clip(lst, max_norm, norms, out)
    keep = torch.from_numpy(covered).to(DEV)
    assert torch.equal(out[:, keep], first[:, keep]) and torch.equal(norms, first_norms)   # bitwise repeatable
    return lst


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 2, 5])
def test_clip_gathers_ragged_lists(src, dst, shift):
    sizes = [1, 7, 64, 1023, 8192, 0, 8193, 3, 30_001]
    nodes = _nodes(3, sizes, [src] * len(sizes), 11 + shift, shift)
    for i, node in enumerate(nodes):                                   # one node below the limit, two above
        for t in node:
            t.mul_(0.1 + i)
    _check_clip(nodes, None, 0.1, dst)
    gapped, at = [], 3
    for k in sizes:
        gapped.append(at)
        at += k + 5
    _check_clip(nodes, gapped, 0.1, dst, columns_extra=9)


def test_clip_mixed_types_and_order_of_columns():
    """fp32 and bf16 tensors in one list, stacked in another order than listed, every tensor on an 8-column boundary."""
    nodes = _nodes(5, [4096, 24, 12_345, 8, 2], ["bf16", "f32", "bf16", "f32", "bf16"], 3)
    _check_clip(nodes, [16_384, 8, 32, 0, 24_000], 0.05, "f32")


# nodes above 262144 elements take other kernels: fewer pieces than CTAs, many more, every type and misalignment
@pytest.mark.parametrize("src,dst,shift", [("f32", "f32", 0), ("f32", "f32", 3), ("bf16", "bf16", 0), ("bf16", "bf16", 5),
                                           ("bf16", "f32", 1), ("f32", "bf16", 2), ("bf16", "f32", 0), ("f32", "bf16", 0)])
@pytest.mark.parametrize("n,sizes", [(1, [300_001]), (3, [1, 270_000, 0, 9, 20_001]), (2, [1_500_000, 3, 700_001]), (40, [262_145])])
def test_clip_of_large_nodes(src, dst, shift, n, sizes):
    nodes = _nodes(n, sizes, [src] * len(sizes), 21 + shift, shift)
    for node in nodes[::2]:
        for t in node:
            t.mul_(0.01)
    lst = _check_clip(nodes, None, 0.1, dst)
    if src == dst:                                                     # the same in place
        from paper_2104_11981_b200 import binding as B
        norms, out = torch.empty(n, device=DEV), torch.empty((n, lst.columns), device=DEV, dtype=TYPE[dst])
        B.gradient_clip(lst, 0.1, norms, out)
        B.gradient_clip(lst, 0.1, norms)
        assert all(torch.equal(torch.cat(node), row) for node, row in zip(nodes, out))


def test_large_nodes_of_mixed_types():
    from paper_2104_11981_b200 import binding as B
    nodes = _nodes(3, [200_003, 17, 100_000, 64], ["bf16", "f32", "f32", "bf16"], 31, 1)
    lst = _check_clip(nodes, [7, 400_000, 200_100, 300_200], 0.2, "f32")
    _check_clip(nodes, None, 0.2, "bf16")
    before, norms = [[to64(t) for t in node] for node in nodes], torch.empty(3, device=DEV)
    B.gradient_clip(lst, 0.2, norms)
    for node, old in zip(nodes, before):
        s = min(1.0, 0.2 / (np.sqrt(sum((x ** 2).sum() for x in old)) + 1e-6))
        for t, x, typ in zip(node, old, ["bf16", "f32", "f32", "bf16"]):
            assert np.all(np.abs(to64(t) - s * x) <= np.abs(s * x) * 24 * U + half_unit(typ, s * x) + 1e-45)


@pytest.mark.parametrize("n,sizes", [(1, [1]), (1, [2_000_003]), (64, [5]), (2, [0, 0]), (300, [17, 300]), (2, [3] * 500),
                                     (5, [400_000, 7]), (700, [262_150])])
def test_norm_over_shapes_and_kinds(n, sizes):
    from paper_2104_11981_b200 import binding as B
    nodes = _nodes(n, sizes, ["f32"] * len(sizes), 5)
    lst = B.gradients_build(nodes)
    norms = torch.full((n,), float("nan"), device=DEV)
    for _ in range(2):
        B.gradient_norm(lst, norms)
        for i in range(n):
            want = _norm64(nodes[i])
            assert abs(float(norms[i]) - want) <= 20 * U * want
    B.gradient_norm(lst, norms, kind=B.NORM_MAX)
    for i in range(n):
        want = max([float(t.abs().max()) for t in nodes[i] if t.numel()], default=0.0)
        assert float(norms[i]) == want


@pytest.mark.parametrize("shift", [0, 3])
@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_clip_in_place(typ, shift):
    from paper_2104_11981_b200 import binding as B
    nodes = _nodes(4, [100, 20_001, 9], [typ] * 3, 9, shift)
    for t in nodes[1]:
        t.mul_(1e-3)                                                   # this node stays below the limit
    before = [[t.clone() for t in node] for node in nodes]
    lst, norms = B.gradients_build(nodes), torch.empty(4, device=DEV)
    gathered = torch.empty((4, lst.columns), device=DEV, dtype=TYPE[typ])
    B.gradient_clip(lst, 0.01, norms, gathered)
    B.gradient_clip(lst, 0.01, norms)
    torch.cuda.synchronize()
    for i in range(4):
        assert torch.equal(torch.cat(nodes[i]), gathered[i])           # the two forms round alike
    assert all(torch.equal(a, b) for a, b in zip(nodes[1], before[1]))
    B.gradient_clip(lst, 0.02, norms, kind=B.NORM_MAX)                 # nothing is above that any more
    assert all(torch.equal(torch.cat(nodes[i]), gathered[i]) for i in range(4))


def test_clip_of_views_of_the_stacked_rows():
    """Gradients written straight into the stacked array are clipped in place; a list gathered into the other columns of
    the same array may share it."""
    from paper_2104_11981_b200 import binding as B
    g = torch.empty((3, 5000), device=DEV).normal_(generator=_gen(2))
    want = to64(g)
    lst = B.gradients_build([[g[i, 8:1000], g[i, 1000:4097]] for i in range(3)])
    norms = torch.empty(3, device=DEV)
    B.gradient_clip(lst, 1.0, norms)
    scale = 1.0 / (np.sqrt((want[:, 8:4097] ** 2).sum(1)) + 1e-6)
    want[:, 8:4097] *= scale[:, None]
    assert np.all(np.abs(to64(g) - want) <= 24 * U * np.abs(want))
    with pytest.raises(B.DecentlamError) as e:
        B.gradient_clip(lst, 1.0, norms, g)
    assert e.value.status == -4
    small = B.gradients_build([[g[i, 4200:4300]] for i in range(3)])
    B.gradient_clip(small, 1.0, norms, g[:, :100])
    assert torch.isfinite(g).all()


@pytest.mark.parametrize("d", [20_000, 300_000])
def test_norm_over_the_whole_range_of_fp32(d):
    """Squares that overflow or vanish in fp32 do not reach the norm; a NaN or an infinity does, in its node alone."""
    from paper_2104_11981_b200 import binding as B
    n = 7
    g = torch.empty((n, d), device=DEV).normal_(generator=_gen(4))
    g[0] *= 1e30
    g[1] *= 1e-30
    g[2] = 0.0
    g[3, 777] = float("inf")
    g[4, 19_999] = float("nan")
    g[5] *= 1e-42                                                      # subnormal
    lst = B.gradients_build([[g[i]] for i in range(n)])
    norms, out = torch.empty(n, device=DEV), torch.empty((n, d), device=DEV)
    B.gradient_clip(lst, 1.0, norms, out)
    got = to64(norms)
    for i in (0, 1, 2, 5, 6):
        want = float(np.sqrt((to64(g[i]) ** 2).sum()))
        assert abs(got[i] - want) <= 20 * U * want + 2e-45
    assert got[3] == np.inf and np.isnan(got[4])
    assert torch.isnan(out[3, 777]) and bool((out[3, :777] == 0).all())            # s = 0, and 0 * inf
    assert torch.isnan(out[4]).all()
    assert torch.equal(out[1], g[1]) and torch.equal(out[2], g[2]) and torch.equal(out[5], g[5])   # s = 1
    for i in (0, 6):
        want = to64(g[i]) / (float(np.sqrt((to64(g[i]) ** 2).sum())) + 1e-6)
        assert np.all(np.abs(to64(out[i]) - want) <= 24 * U * np.abs(want))
    B.gradient_norm(lst, norms, kind=B.NORM_MAX)
    got = to64(norms)
    assert got[3] == np.inf and np.isnan(got[4]) and got[0] == float(g[0].abs().max())


@pytest.mark.parametrize("size", [70_000, 400_000])
def test_streams_and_graphs(size):
    """On another stream than the current one, and captured: the replay follows the tensors' contents."""
    from paper_2104_11981_b200 import binding as B
    nodes = _nodes(2, [size, 33], ["f32", "f32"], 8)
    lst = B.gradients_build(nodes)
    norms, out = torch.empty(2, device=DEV), torch.empty((2, lst.columns), device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.gradient_clip(lst, 0.05, norms, out, stream=side)
    side.synchronize()
    eager, eager_norms = out.clone(), norms.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.gradient_clip(lst, 0.05, norms, out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, eager) and torch.equal(norms, eager_norms)
    for node in nodes:
        for t in node:
            t.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(norms, 2.0 * eager_norms)


def test_refusals():
    from paper_2104_11981_b200 import binding as B
    nodes = _nodes(2, [100, 50], ["f32", "bf16"], 1)
    lst = B.gradients_build(nodes)
    norms, out = torch.empty(2, device=DEV), torch.empty((2, 150), device=DEV)
    vp, lib = ctypes.c_void_p, B.raw()

    def clip(handle=lst.handle, kind=0, limit=1.0, pn=norms.data_ptr(), g=out.data_ptr(), gd=0, ldg=150):
        return lib.gradient_clip(handle, kind, limit, vp(pn), vp(g), gd, ldg, None)

    before = B.launch_count()
    assert clip(handle=None) == -1 and clip(pn=0) == -1
    assert clip(kind=2) == -6 and clip(gd=5) == -6
    assert clip(limit=0.0) == -5 and clip(limit=float("nan")) == -5 and clip(limit=float("inf")) == -5
    assert clip(ldg=149) == -2
    assert clip(g=out.data_ptr() + 2) == -3 and clip(pn=norms.data_ptr() + 1) == -3
    assert clip(g=nodes[0][0].data_ptr()) == -4 and clip(pn=nodes[1][0].data_ptr()) == -4
    assert clip(pn=out.data_ptr() + 4) == -4
    assert lib.gradient_norm(lst.handle, 0, None, None) == -1
    assert B.launch_count() == before
    assert clip() == 0
    torch.cuda.synchronize()
