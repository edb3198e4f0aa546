"""Training operators without a GPU: the layout of gradient lists, and the refusal of bad arguments before anything is
launched (pointers are never read by these calls)."""
import ctypes

import pytest

from paper_2104_11981_b200 import binding as B

vp, i64 = ctypes.c_void_p, ctypes.c_int64


def _build(n=2, sizes=(10, 6), dtypes=(0, 0), data=None, offsets=None, out=True):
    t = len(sizes)
    data = data if data is not None else [4096 * (1 + k) for k in range(n * t)]
    handle = vp()
    rc = B.raw().gradients_build(n, t, (i64 * t)(*sizes), (ctypes.c_int * t)(*dtypes), (vp * len(data))(*data),
                                 (i64 * t)(*offsets) if offsets is not None else None, ctypes.byref(handle) if out else None)
    if rc != 0:
        assert not handle.value
    return rc, handle


def test_gradient_list_refusals():
    assert _build(out=False)[0] == -1
    assert _build(n=0, data=[])[0] == -2
    assert _build(n=B.MAX_NODES + 1, data=[16] * (2 * B.MAX_NODES + 2))[0] == -8
    assert _build(sizes=(10, -1))[0] == -2
    assert _build(dtypes=(0, 3))[0] == -6
    assert _build(data=[4096, 0, 8192, 12288])[0] == -1
    assert _build(data=[4096, 8193, 16384, 20480])[0] == -3
    assert _build(data=[4096, 4096 + 36, 16384, 20480])[0] == -4            # node 0's tensors share an element
    assert _build(offsets=(0, 9))[0] == -4 and _build(offsets=(0, -1))[0] == -2


def test_gradient_list_layout():
    import torch
    if torch.cuda.is_available():
        pytest.skip("host-only handles exist without a CUDA device")
    rc, h = _build(sizes=(10, 0, 6), dtypes=(0, 1, 1), data=[4096, 0, 8192, 12288, 0, 16384])
    assert rc == 0
    lst = B.Gradients(h, 2, 3, None)
    assert lst.offsets == [0, 10, 10] and lst.columns == 16
    rc, h = _build(offsets=(32, 8))
    lst = B.Gradients(h, 2, 2, None)
    assert rc == 0 and lst.offsets == [32, 8] and lst.columns == 42
    assert B.raw().gradient_norm(h, 0, vp(1 << 20), None) == -9             # no device
    assert B.raw().gradients_layout(None, None, None) == -1
    assert B.raw().gradients_destroy(None) == 0


def _norm(**kw):
    a = dict(n=2, rows=3, c=8, x=0x10000, dt=0, ldx=8, w=0x20000, ldw=8, b=0x30000, ldb=8, eps=1e-5, y=0x40000, ldy=8,
             mean=0x50000, rstd=0x60000)
    a.update(kw)
    return B.raw().layer_norm(a["n"], a["rows"], a["c"], vp(a["x"]), a["dt"], a["ldx"], vp(a["w"]), a["ldw"], vp(a["b"]),
                              a["ldb"], a["eps"], vp(a["y"]), a["ldy"], vp(a["mean"]), vp(a["rstd"]), None)


def test_layer_norm_refusals():
    for name in ("x", "w", "y", "mean", "rstd"):
        assert _norm(**{name: 0}) == -1, name
    assert _norm(n=0) == -2 and _norm(rows=-1) == -2 and _norm(c=0) == -2
    assert _norm(n=B.MAX_NODES + 1) == -8 and _norm(rows=1 << 50) == -8
    assert _norm(ldx=7) == -2 and _norm(ldy=7) == -2 and _norm(ldw=7) == -2 and _norm(ldb=7) == -2
    assert _norm(dt=2) == -6
    assert _norm(x=0x10002) == -3 and _norm(y=0x40001, dt=1) == -3 and _norm(w=0x20002) == -3 and _norm(mean=0x50002) == -3
    assert _norm(eps=-1.0) == -5 and _norm(eps=float("nan")) == -5
    assert _norm(y=0x10004) == -4 and _norm(y=0x20000) == -4 and _norm(mean=0x60004) == -4 and _norm(rstd=0x10000) == -4
    assert _norm(y=0x10000, ldy=9) == -4                                     # in place needs the same stride
    assert _norm(rows=0) == 0


def _norm_grad(**kw):
    a = dict(n=2, rows=3, c=8, x=0x10000, dt=0, ldx=8, dy=0x20000, ldy=8, w=0x30000, ldw=8, mean=0x40000, rstd=0x50000,
             dx=0x60000, lddx=8, gw=0x70000, ldgw=8, gb=0x80000, ldgb=8, gt=0, ws=0x90000, wb=1 << 14)
    a.update(kw)
    return B.raw().layer_norm_grad(a["n"], a["rows"], a["c"], vp(a["x"]), a["dt"], a["ldx"], vp(a["dy"]), a["ldy"], vp(a["w"]),
                                   a["ldw"], vp(a["mean"]), vp(a["rstd"]), vp(a["dx"]), a["lddx"], vp(a["gw"]), a["ldgw"],
                                   vp(a["gb"]), a["ldgb"], a["gt"], vp(a["ws"]), a["wb"], None)


def test_layer_norm_grad_refusals():
    for name in ("x", "dy", "w", "mean", "rstd", "dx", "gw"):
        assert _norm_grad(**{name: 0}) == -1, name
    assert _norm_grad(n=0) == -2 and _norm_grad(ldgw=7) == -2 and _norm_grad(ldgb=7) == -2 and _norm_grad(lddx=7) == -2
    assert _norm_grad(dt=2) == -6 and _norm_grad(gt=7) == -6
    assert _norm_grad(dx=0x60001, dt=1) == -3 and _norm_grad(gw=0x70002) == -3
    need = B.layer_norm_grad_workspace_bytes(2, 3, 8)
    assert need >= 2 * 3 * 2 * 8 * 4
    assert _norm_grad(wb=need - 1) == -10 and _norm_grad(ws=0) == -10 and _norm_grad(ws=0x90010) == -10
    assert _norm_grad(dx=0x10010) == -4 and _norm_grad(gw=0x80004) == -4 and _norm_grad(gw=0x10000) == -4
    assert _norm_grad(ws=0x70000) == -4 and _norm_grad(gb=0x30000) == -4 and _norm_grad(dx=0x40000) == -4
    # the columns of one stacked array may be weight and bias gradients; a column too many meets the neighbour's
    assert _norm_grad(gw=0x70000, gb=0x70000 + 28, ldgw=16, ldgb=16) == -4
    with pytest.raises(B.DecentlamError) as e:
        B.layer_norm_grad_workspace_bytes(0, 1, 1)
    assert e.value.status == -2


def _policy(**kw):
    a = dict(n=2, rows=3, v=100, z=0x10000, dt=0, ldl=100, tok=0x20000, w=0x30000, adv=0x40000, old=0x50000, ref=0x60000,
             lo=0.2, hi=0.2, kl=0.1, loss=0x70000, logp=0x80000, d=0x90000, ldd=100, ws=0xa0000, wb=256)
    a.update(kw)
    return B.raw().policy_loss_grad(a["n"], a["rows"], a["v"], vp(a["z"]), a["dt"], a["ldl"], vp(a["tok"]), vp(a["w"]),
                                    vp(a["adv"]), vp(a["old"]), vp(a["ref"]), a["lo"], a["hi"], a["kl"], vp(a["loss"]),
                                    vp(a["logp"]), vp(a["d"]), a["ldd"], vp(a["ws"]), a["wb"], None)


def test_policy_loss_refusals():
    for name in ("z", "tok", "w", "adv", "old", "loss", "logp"):
        assert _policy(**{name: 0}) == -1, name
    assert _policy(ref=0) == -5                                              # a KL term needs its reference
    assert _policy(n=0) == -2 and _policy(v=0) == -2 and _policy(ldl=99) == -2 and _policy(ldd=99) == -2
    assert _policy(v=1 << 40) == -8 and _policy(rows=1 << 31) == -8
    assert _policy(dt=9) == -6
    assert _policy(tok=0x20004) == -3 and _policy(z=0x10001, dt=1) == -3 and _policy(w=0x30001) == -3
    assert _policy(lo=-0.1) == -5 and _policy(hi=float("nan")) == -5 and _policy(kl=float("inf")) == -5
    assert _policy(ws=0) == -10 and _policy(wb=255) == -10 and _policy(ws=0xa0080) == -10
    assert _policy(d=0x10004) == -4 and _policy(loss=0x30000) == -4 and _policy(logp=0x10000) == -4
    assert _policy(ws=0x20000) == -4 and _policy(d=0x10000, ldd=101) == -4


def test_calls_convert_their_arguments():
    from paper_2104_11981_b200 import _calls
    none = [1, 1, 8, None, 0, 8, None, 8, None, 8, 1e-5, None, 8, None, None, 0]
    assert _calls.layer_norm(*none) == B._lib.layer_norm(*none) == -1  # None is a null pointer in both
    for bad in (none[:-1], none + [0], [None if k == 10 else v for k, v in enumerate(none)], ["1"] + none[1:]):
        with pytest.raises(TypeError):
            _calls.layer_norm(*bad)
    with pytest.raises(OverflowError):
        _calls.layer_norm(1, 1 << 64, *none[2:])
    assert _calls.layer_norm(1, 1 << 62, *none[2:]) == B._lib.layer_norm(1, 1 << 62, *none[2:])  # 64-bit lengths arrive whole
