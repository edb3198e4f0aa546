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
