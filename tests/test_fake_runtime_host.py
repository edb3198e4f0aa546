"""Host side of the library on a CUDA runtime that is not one (fake_cuda_runtime.cpp): what reaches the device before a handle is handed
out, and what is left behind when the runtime fails."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2104_11981_b200", "csrc")
vp, i64, c_int = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake") / "libhost.so")
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    sources = [os.path.join(CSRC, s) for s in ("topology.cpp", "sharded.cpp", "gradients.cpp", "train.cpp")]
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    "-I", os.path.join(cuda, "include"), os.path.join(ROOT, "tests", "fake_cuda_runtime.cpp"), *sources, "-o", out],
                   check=True)
    return ctypes.CDLL(out)


def _gradients(lib, sizes=(300_000, 10)):
    t = len(sizes)
    data = (vp * (2 * t))(*[(1 + k) << 24 for k in range(2 * t)])
    handle = vp()
    rc = lib.gradients_build(2, t, (i64 * t)(*sizes), (c_int * t)(*([0] * t)), data, None, ctypes.byref(handle))
    return rc, handle


def _topology(lib, n=8):
    handle = vp()
    return lib.topology_build(0, n, None, None, None, ctypes.byref(handle)), handle


def _shard(lib, topo):
    handle = vp()
    return lib.topology_shard(topo, 0, 2, ctypes.byref(handle)), handle


def test_tables_have_reached_the_device_when_the_handle_is_handed_out(lib):
    """A first call may come on a stream that nothing orders behind the copies."""
    for build, destroy in ((lambda: _gradients(lib), lib.gradients_destroy), (lambda: _topology(lib), lib.topology_destroy)):
        before = lib.fake_copies()
        rc, handle = build()
        assert rc == 0 and lib.fake_copies() > before and lib.fake_staged() == 0
        assert destroy(handle) == 0
    rc, topo = _topology(lib)
    before = lib.fake_copies()
    rc, shard = _shard(lib, topo)
    assert rc == 0 and lib.fake_copies() > before and lib.fake_staged() == 0
    assert lib.topology_shard_destroy(shard) == 0 and lib.topology_destroy(topo) == 0
    assert lib.fake_blocks() == 0


def test_a_build_that_runs_out_of_memory_leaves_nothing_behind(lib):
    """Neither memory nor the runtime's last error, which the next step's launch would report as its own."""
    for k in range(4):
        lib.fake_mallocs_left(k)
        rc, handle = _gradients(lib)
        lib.fake_mallocs_left(-1)
        assert (rc, bool(handle.value)) == ((-9, False) if k < 3 else (0, True))   # pieces, scales, partial sums
        assert lib.fake_last_error() == 0
        lib.gradients_destroy(handle)
        assert lib.fake_blocks() == 0


def test_a_launch_that_fails_leaves_no_error_behind(lib):
    rc, handle = _gradients(lib)
    assert rc == 0
    flt, at = ctypes.c_float, lambda k: vp(k << 16)
    calls = {
        "gradient_norm": (handle, 0, vp(1 << 20), None),
        "gradient_clip": (handle, 0, flt(1.0), vp(1 << 20), None, 0, i64(0), None),
        "layer_norm": (2, i64(3), i64(8), at(1), 0, i64(8), at(2), i64(8), at(3), i64(8), flt(1e-5), at(4), i64(8), at(5), at(6), None),
        "layer_norm_grad": (2, i64(3), i64(8), at(1), 0, i64(8), at(2), i64(8), at(3), i64(8), at(4), at(5), at(6), i64(8), at(7),
                            i64(8), at(8), i64(8), 0, at(9), i64(1 << 14), None),
        "policy_loss_grad": (2, i64(3), i64(100), at(1), 0, i64(100), at(2), at(3), at(4), at(5), at(6), flt(0.2), flt(0.2), flt(0.1),
                             at(7), at(8), at(9), i64(100), at(10), i64(256), None)}
    for fail in (1, 0):
        lib.fake_launches_fail(fail)
        for name, args in calls.items():
            assert getattr(lib, name)(*args) == (-9 if fail else 0), name
            assert lib.fake_last_error() == 0, name
    lib.gradients_destroy(handle)


def test_row_strides_of_the_gathered_rows_are_bounded(lib):
    """A stride whose rows' addresses wrap would pass the overlap checks; none above 2^42 elements in all can exist."""
    rc, handle = _gradients(lib)
    assert rc == 0
    for ldg, want in ((300_009, -2), (300_010, 0), (1 << 41, 0), ((1 << 41) + 1, -8), (1 << 61, -8), ((1 << 63) - 1, -8)):
        assert lib.gradient_clip(handle, 0, ctypes.c_float(1.0), vp(1 << 20), vp(1 << 40), 0, i64(ldg), None) == want, ldg
    lib.gradients_destroy(handle)


def test_a_policy_loss_without_rows_needs_no_reference(lib):
    """Tensors without elements have no address, the reference's among them."""
    lib.fake_launches_fail(0)
    flt, none = ctypes.c_float, vp(None)

    def call(rows, ref):
        at = (lambda k: vp(k << 16)) if rows else (lambda k: none)
        return lib.policy_loss_grad(2, i64(rows), i64(100), at(1), 0, i64(100), at(2), at(3), at(4), at(5), ref, flt(0.2), flt(0.2), flt(0.1),
                                    vp(7 << 16), at(8), at(9), i64(100), vp(10 << 16), i64(256), None)
    assert call(3, vp(6 << 16)) == 0 and call(3, none) == -5 and call(0, none) == 0
