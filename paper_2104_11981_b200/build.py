"""Build libdecentlam.so (CUDA kernels + C ABI) for sm_100a and _calls (its CPython entry points), in-tree.

Usage: python -m paper_2104_11981_b200.build [--force] [--verbose]
nvcc cross-compiles without a GPU; the runtime is linked statically so the library loads
(and its host-only entry points work) on machines without a CUDA device.  Every source is
compiled to an object of its own (in parallel, only when it or a header changed), then linked.
"""
import importlib.util
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
OBJ = os.path.join(HERE, "_build")
OUT = os.path.join(HERE, "libdecentlam.so")
CALLS = os.path.join(HERE, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))
SOURCES = ["api.cpp", "topology.cpp", "sharded.cpp", "step_kernels.cu", "step_merged.cu", "step_sharded.cu",
           "pmsgd_kernel.cu", "lsq_kernels.cu", "gradients.cpp", "gradient_kernels.cu", "train.cpp", "layer_norm.cu",
           "policy_loss.cu", "model.cpp", "embedding.cu", "rms_norm.cu", "dropout.cu", "logits.cu"]
ARCH = ["-gencode", "arch=compute_100a,code=sm_100a"]


def _headers():
    return [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))] + \
           [os.path.join(INCLUDE, "decentlam.h")]


def _stale() -> bool:
    if not os.path.exists(OUT):
        return True
    t = os.path.getmtime(OUT)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + _headers()
    return any(os.path.getmtime(p) > t for p in deps)


def _compile(src: str, force: bool, verbose: bool) -> str:
    obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    path = os.path.join(CSRC, src)
    if not force and os.path.exists(obj):
        t = os.path.getmtime(obj)
        if all(os.path.getmtime(p) <= t for p in [path] + _headers()):
            return obj
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc] + ARCH + ["-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
                           "-I", INCLUDE, "-I", CSRC, "-x", "cu", "-c", path, "-o", obj]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    subprocess.run(cmd, check=True)
    return obj


def _exchange_flags():
    """Flags for reading tensors through their exchange interface, whose header comes with them; none where that header is missing or
    older than what the module uses of it, and the binding reads tensors itself."""
    spec = importlib.util.find_spec("torch")
    include = os.path.join(os.path.dirname(spec.origin), "include") if spec and spec.origin else ""
    header = os.path.join(include, "ATen", "dlpack.h")
    if not os.path.exists(header):
        return []
    with open(header, encoding="utf-8") as f:
        text = f.read()
    used = ("DLPackExchangeAPI;", "dltensor_from_py_object_no_sync;", "current_work_stream;", "prev_api;", "kDLFloat8_e4m3fn")
    return ["-DDLM_TENSORS", "-isystem", include] if all(name in text for name in used) else []


def _build_calls(force: bool) -> None:
    src = os.path.join(CSRC, "calls.c")
    if not force and os.path.exists(CALLS) and all(os.path.getmtime(p) <= os.path.getmtime(CALLS)
                                                   for p in (src, os.path.join(INCLUDE, "decentlam.h"))):
        return
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        print("Python.h not found: _calls is left out, the binding calls through ctypes", file=sys.stderr)
        return
    tmp = CALLS + ".tmp"
    more = _exchange_flags()
    subprocess.run([os.environ.get("CC", "gcc"), "-O2", "-fPIC", "-shared", *more, "-I", INCLUDE, "-I", sysconfig.get_paths()["include"],
                    src, "-o", tmp, "-L", HERE, "-l:libdecentlam.so", "-Wl,-rpath,$ORIGIN"], check=True)
    os.replace(tmp, CALLS)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        _build_calls(force)
        return OUT
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as pool:
        objs = list(pool.map(lambda s: _compile(s, force, verbose), SOURCES))
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = OUT + ".tmp"
    subprocess.run([nvcc] + ARCH + ["-shared", "-Xcompiler", "-fPIC", "-cudart", "static"] + objs + ["-o", tmp], check=True)
    os.replace(tmp, OUT)
    _build_calls(force)
    return OUT


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
