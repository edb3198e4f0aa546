"""Operators between tokens and logits without a GPU: the refusal of bad arguments before anything is launched (pointers are never
read by these calls), and the generator's definition against its authors' known answers."""
import ctypes

import numpy as np
import pytest

from helpers_philox import philox_4x32_10
from paper_2104_11981_b200 import binding as B

vp = ctypes.c_void_p
NAN, INF = float("nan"), float("inf")


def test_generator_known_answers():
    """The three vectors for philox4x32-10 that its authors publish with their generators."""
    for counter, key, want in (((0,) * 4, (0,) * 2, (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
                               ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
                               ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
                                (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        got = philox_4x32_10([np.array([v], dtype=np.uint64) for v in counter], key)
        assert tuple(int(v[0]) for v in got) == want


def _embedding(**kw):
    a = dict(n=2, rows=3, v=10, c=8, t=0x10000, tt=0, ldt=80, tok=0x20000, s=1.0, y=0x30000, dt=0, ldy=8)
    a.update(kw)
    return B.raw().embedding(a["n"], a["rows"], a["v"], a["c"], vp(a["t"]), a["tt"], a["ldt"], vp(a["tok"]), a["s"], vp(a["y"]),
                             a["dt"], a["ldy"], None)


def test_embedding_refusals():
    for name in ("t", "tok", "y"):
        assert _embedding(**{name: 0}) == -1, name
    assert _embedding(n=0) == -2 and _embedding(rows=-1) == -2 and _embedding(v=0) == -2 and _embedding(c=0) == -2
    assert _embedding(ldt=79) == -2 and _embedding(ldy=7) == -2
    assert _embedding(n=B.MAX_NODES + 1) == -8 and _embedding(v=1 << 31) == -8 and _embedding(rows=1 << 40) == -8
    assert _embedding(c=1 << 40) == -8 and _embedding(ldt=1 << 50) == -8
    assert _embedding(dt=2) == -6 and _embedding(tt=-1) == -6
    assert _embedding(t=0x10002) == -3 and _embedding(tok=0x20004) == -3 and _embedding(y=0x30001, dt=1) == -3
    assert _embedding(s=NAN) == -5 and _embedding(s=INF) == -5
    assert _embedding(y=0x10010) == -4 and _embedding(y=0x20000 - 32) == -4
    assert _embedding(rows=0) == 0


def _embedding_grad(**kw):
    a = dict(n=2, rows=3, v=10, c=8, tok=0x20000, dy=0x30000, dt=0, ldy=8, s=1.0, add=0, g=0x40000, gt=0, ldg=80, ws=0x80000, wb=1 << 16)
    a.update(kw)
    return B.raw().embedding_grad(a["n"], a["rows"], a["v"], a["c"], vp(a["tok"]), vp(a["dy"]), a["dt"], a["ldy"], a["s"], a["add"],
                                  vp(a["g"]), a["gt"], a["ldg"], vp(a["ws"]), a["wb"], None)


def test_embedding_grad_refusals():
    for name in ("tok", "dy", "g"):
        assert _embedding_grad(**{name: 0}) == -1, name
    assert _embedding_grad(ldy=7) == -2 and _embedding_grad(ldg=79) == -2 and _embedding_grad(v=-1) == -2
    assert _embedding_grad(dt=5) == -6 and _embedding_grad(gt=2) == -6 and _embedding_grad(add=2) == -6
    assert _embedding_grad(g=0x40002) == -3 and _embedding_grad(dy=0x30002) == -3 and _embedding_grad(tok=0x20001) == -3
    assert _embedding_grad(s=NAN) == -5
    need = B.embedding_grad_workspace_bytes(2, 3, 10, 8)
    assert need >= 2 * 3 * 8 and _embedding_grad(wb=need - 1) == -10 and _embedding_grad(ws=0) == -10 and _embedding_grad(ws=0x80010) == -10
    assert _embedding_grad(g=0x30000 - 16) == -4 and _embedding_grad(g=0x20000) == -4 and _embedding_grad(ws=0x40000) == -4
    assert _embedding_grad(ws=0x30000) == -4
    with pytest.raises(B.DecentlamError) as e:
        B.embedding_grad_workspace_bytes(1, 1, 0, 1)
    assert e.value.status == -2
    # workspaces grow with the text and stay far below the gradient's size
    assert B.embedding_grad_workspace_bytes(8, 2048, 32_768, 1024) < 8 * 32_768 * 1024 * 4 // 16


def _rms(**kw):
    a = dict(n=2, rows=3, c=8, x=0x10000, dt=0, ldx=8, r=0x20000, ldr=8, w=0x30000, ldw=8, eps=1e-5, h=0x40000, ldh=8, y=0x50000, ldy=8,
             y8=0x60000, ld8=8, sc=0x70000, rstd=0x80000)
    a.update(kw)
    return B.raw().rms_norm(a["n"], a["rows"], a["c"], vp(a["x"]), a["dt"], a["ldx"], vp(a["r"]), a["ldr"], vp(a["w"]), a["ldw"],
                            a["eps"], vp(a["h"]), a["ldh"], vp(a["y"]), a["ldy"], vp(a["y8"]), a["ld8"], vp(a["sc"]), vp(a["rstd"]), None)


def test_rms_norm_refusals():
    for name in ("x", "w", "rstd", "y8", "sc"):                              # 8 bits need scales and the other way about
        assert _rms(**{name: 0}) == -1, name
    assert _rms(y=0, y8=0, sc=0) == -1                                       # no output
    assert _rms(n=0) == -2 and _rms(rows=-1) == -2 and _rms(c=0) == -2
    for name in ("ldx", "ldr", "ldw", "ldh", "ldy", "ld8"):
        assert _rms(**{name: 7}) == -2, name
    assert _rms(n=B.MAX_NODES + 1) == -8 and _rms(rows=1 << 50) == -8 and _rms(ld8=1 << 60) == -8
    assert _rms(dt=2) == -6
    assert _rms(x=0x10002) == -3 and _rms(r=0x20002) == -3 and _rms(h=0x40001, dt=1) == -3 and _rms(rstd=0x80002) == -3
    assert _rms(eps=-1.0) == -5 and _rms(eps=NAN) == -5
    assert _rms(h=0x50004) == -4 and _rms(h=0x10004) == -4 and _rms(y=0x20004) == -4 and _rms(y=0x30000) == -4
    assert _rms(y8=0x10000) == -4 and _rms(rstd=0x70004) == -4 and _rms(sc=0x20000) == -4 and _rms(y=0x10000, ldy=9) == -4
    assert _rms(h=0x10000, y=0x10000) == -4                                  # both in one place
    assert _rms(rows=0) == 0


def _rms_grad(**kw):
    a = dict(n=2, rows=3, c=8, h=0x10000, dt=0, ldh=8, dy=0x20000, ldy=8, r=0x30000, ldr=8, w=0x40000, ldw=8, rstd=0x50000, dh=0x60000,
             lddh=8, gw=0x70000, ldgw=8, gt=0, ws=0x90000, wb=1 << 14)
    a.update(kw)
    return B.raw().rms_norm_grad(a["n"], a["rows"], a["c"], vp(a["h"]), a["dt"], a["ldh"], vp(a["dy"]), a["ldy"], vp(a["r"]), a["ldr"],
                                 vp(a["w"]), a["ldw"], vp(a["rstd"]), vp(a["dh"]), a["lddh"], vp(a["gw"]), a["ldgw"], a["gt"],
                                 vp(a["ws"]), a["wb"], None)


def test_rms_norm_grad_refusals():
    for name in ("h", "dy", "w", "rstd", "dh", "gw"):
        assert _rms_grad(**{name: 0}) == -1, name
    for name in ("ldh", "ldy", "ldr", "ldw", "lddh", "ldgw"):
        assert _rms_grad(**{name: 7}) == -2, name
    assert _rms_grad(dt=2) == -6 and _rms_grad(gt=7) == -6
    assert _rms_grad(dh=0x60001, dt=1) == -3 and _rms_grad(gw=0x70002) == -3 and _rms_grad(r=0x30002) == -3
    need = B.rms_norm_grad_workspace_bytes(2, 3, 8)
    assert need >= 2 * 3 * 8 * 4
    assert _rms_grad(wb=need - 1) == -10 and _rms_grad(ws=0) == -10 and _rms_grad(ws=0x90010) == -10
    assert _rms_grad(dh=0x10010) == -4 and _rms_grad(dh=0x30004) == -4 and _rms_grad(gw=0x10000) == -4 and _rms_grad(gw=0x60000) == -4
    assert _rms_grad(ws=0x70000) == -4 and _rms_grad(gw=0x40000) == -4 and _rms_grad(dh=0x50000) == -4 and _rms_grad(ws=0x30000) == -4


def _dropout(**kw):
    a = dict(n=2, rows=3, c=8, x=0x10000, dt=0, ldx=8, r=0x20000, ldr=8, p=0.5, st=0x30000, site=0, y=0x40000, ldy=8)
    a.update(kw)
    return B.raw().dropout(a["n"], a["rows"], a["c"], vp(a["x"]), a["dt"], a["ldx"], vp(a["r"]), a["ldr"], a["p"], vp(a["st"]), a["site"],
                           vp(a["y"]), a["ldy"], None)


def test_dropout_refusals():
    for name in ("x", "st", "y"):
        assert _dropout(**{name: 0}) == -1, name
    assert _dropout(n=0) == -2 and _dropout(ldx=7) == -2 and _dropout(ldy=7) == -2 and _dropout(ldr=7) == -2
    assert _dropout(rows=1 << 50) == -8 and _dropout(dt=2) == -6
    assert _dropout(x=0x10002) == -3 and _dropout(st=0x30004) == -3 and _dropout(y=0x40001, dt=1) == -3
    assert _dropout(p=-0.1) == -5 and _dropout(p=1.0) == -5 and _dropout(p=NAN) == -5 and _dropout(site=-1) == -5
    assert _dropout(site=1 << 32) == -5
    assert _dropout(y=0x10004) == -4 and _dropout(y=0x20004) == -4 and _dropout(y=0x30000) == -4 and _dropout(y=0x10000, ldy=9) == -4
    assert _dropout(rows=0) == 0


def _logits(**kw):
    a = dict(n=2, rows=3, v=100, z=0x10000, dt=0, ldl=100, b=0x20000, ldb=100, m=0x30000, ldm=4, t=0x40000, tl=20, st=0x50000, rep=0x60000,
             fr=0x70000, pr=0x80000, te=0x90000, o=0xa0000, ldo=100)
    a.update(kw)
    return B.raw().logits_adjust(a["n"], a["rows"], a["v"], vp(a["z"]), a["dt"], a["ldl"], vp(a["b"]), a["ldb"], vp(a["m"]), a["ldm"],
                                 vp(a["t"]), a["tl"], vp(a["st"]), vp(a["rep"]), vp(a["fr"]), vp(a["pr"]), vp(a["te"]), vp(a["o"]),
                                 a["ldo"], None)


def test_logits_adjust_refusals():
    assert _logits(z=0) == -1 and _logits(o=0) == -1
    assert _logits(t=0) == -1 and _logits(st=0) == -1                        # a text and its bounds come together
    assert _logits(t=0, tl=0, st=0) == -1                                    # penalties without texts
    assert _logits(n=0) == -2 and _logits(v=0) == -2 and _logits(ldl=99) == -2 and _logits(ldo=99) == -2 and _logits(ldb=99) == -2
    assert _logits(ldm=3) == -2 and _logits(tl=-1) == -2
    assert _logits(v=1 << 40) == -8 and _logits(rows=1 << 31) == -8 and _logits(ldm=1 << 60) == -8 and _logits(tl=1 << 31) == -8
    assert _logits(dt=9) == -6
    assert _logits(z=0x10001, dt=1) == -3 and _logits(b=0x20002) == -3 and _logits(m=0x30001) == -3 and _logits(t=0x40004) == -3
    assert _logits(st=0x50004) == -3 and _logits(rep=0x60002) == -3 and _logits(te=0x90002) == -3
    for place in (0x10004, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000, 0x70000, 0x80000, 0x90000):
        assert _logits(o=place) == -4, hex(place)
    assert _logits(o=0x10000, ldo=101) == -4
    assert _logits(rows=0) == 0


def _logits_grad(**kw):
    a = dict(n=2, rows=3, v=100, g=0x10000, dt=0, ldg=100, z=0x20000, ldl=100, m=0x30000, ldm=4, t=0x40000, tl=20, st=0x50000, rep=0x60000,
             te=0x90000, o=0xa0000, ldo=100)
    a.update(kw)
    return B.raw().logits_adjust_grad(a["n"], a["rows"], a["v"], vp(a["g"]), a["dt"], a["ldg"], vp(a["z"]), a["ldl"], vp(a["m"]), a["ldm"],
                                      vp(a["t"]), a["tl"], vp(a["st"]), vp(a["rep"]), vp(a["te"]), vp(a["o"]), a["ldo"], None)


def test_logits_adjust_grad_refusals():
    assert _logits_grad(g=0) == -1 and _logits_grad(o=0) == -1 and _logits_grad(z=0) == -1 and _logits_grad(st=0) == -1
    assert _logits_grad(ldg=99) == -2 and _logits_grad(ldl=99) == -2 and _logits_grad(ldo=99) == -2
    assert _logits_grad(dt=-3) == -6 and _logits_grad(z=0x20002) == -3 and _logits_grad(o=0xa0002) == -3
    assert _logits_grad(o=0x10004) == -4 and _logits_grad(o=0x20004) == -4 and _logits_grad(o=0x60000) == -4
    assert _logits_grad(rows=0) == 0


def test_calls_convert_their_arguments():
    from paper_2104_11981_b200 import _calls
    big = 1 << 20
    for name, args, want in (
            ("embedding", [2, 3, 10, 8, big, 0, 79, 2 * big, 1.0, 3 * big, 0, 8, 0], -2),
            ("embedding_grad", [2, 3, 10, 8, big, 2 * big, 0, 8, 1.0, 0, 3 * big, 0, 80, 4 * big, 1, 0], -10),
            ("rms_norm", [2, 3, 8, big, 0, 8, None, 0, 2 * big, 8, -1.0, None, 0, 3 * big, 8, None, 0, None, 4 * big, 0], -5),
            ("rms_norm_grad", [2, 3, 8, big, 0, 8, big, 8, None, 0, 2 * big, 8, 3 * big, 4 * big, 8, 5 * big, 8, 3, 6 * big, 1, 0], -6),
            ("dropout", [2, 3, 8, big, 0, 8, None, 0, 2.0, 2 * big, 0, 3 * big, 8, 0], -5),
            ("logits_adjust", [2, 3, 8, big, 0, 8, None, 0, None, 0, None, 0, None, big, None, None, None, 2 * big, 8, 0], -1),
            ("logits_adjust_grad", [2, 3, 8, big, 0, 8, None, 0, None, 0, None, 0, None, None, None, 2 * big, 7, 0], -2)):
        assert getattr(_calls, name)(*args) == getattr(B._lib, name)(*args) == want, name
        with pytest.raises(TypeError):
            getattr(_calls, name)(*args[:-1])
        with pytest.raises(OverflowError):
            getattr(_calls, name)(args[0], 1 << 64, *args[2:])
        assert getattr(_calls, name)(1 << 40, *args[1:]) == getattr(B._lib, name)(1 << 40, *args[1:]) == -8  # not cut to 32 bits


def test_binding_refuses_tensors_without_a_device():
    import torch
    x = torch.zeros((1, 2, 8))
    with pytest.raises((AssertionError, RuntimeError)):
        B.dropout(x, 0.1, torch.zeros(2, dtype=torch.int64), x)
    with pytest.raises((AssertionError, RuntimeError)):
        B.rms_norm(x, torch.ones((1, 8)), 1e-5, x.clone(), torch.zeros((1, 2)))


def test_calls_without_a_device_fail():
    """Nothing divides by a device's properties, nothing is read: arguments that are right end with the CUDA status."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("for machines without a CUDA device")
    assert _embedding() == _embedding_grad() == _embedding_grad(rows=300, wb=1 << 20) == _rms() == _rms(y8=0, sc=0) == -9
    assert _rms_grad() == _dropout() == _dropout(ldx=9) == _logits() == _logits(v=5000, ldl=5000, ldo=5000, ldb=5000, ldm=200, z=0x100000,
                                                                                    o=0x200000, b=0x300000, m=0x400000) == _logits_grad() == -9
