"""The library is used from any Python: without the CPython module of the training operators' calls, ctypes makes them."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = """
import sys
sys.path.insert(0, %r)
if %r:
    sys.modules["paper_2104_11981_b200._calls"] = None                    # as if it had not been built
from paper_2104_11981_b200 import binding as B
assert ("ctypes" in type(B._calls).__module__) == %r
big = 1 << 20
print(B._calls.gradient_norm(None, 0, big, 0), B._calls.gradient_clip(None, 0, 1, None, None, 0, 0, 0))
print(B._calls.layer_norm(2, 3, 8, big, 0, 8, 2 * big, 8, None, 0, -1.0, 3 * big, 8, 4 * big, 5 * big, 0),
      B._calls.layer_norm(2, 1 << 50, 8, big, 0, 8, 2 * big, 8, None, 0, 1e-5, 3 * big, 8, 4 * big, 5 * big, 0))
print(B._calls.layer_norm_grad(2, 3, 8, big, 0, 8, big, 7, big, 8, big, big, big, 8, big, 8, None, 0, 0, big, big, 0))
print(B._calls.policy_loss_grad(2, 3, 100, big, 5, 100, big, big, big, big, None, 0.2, 0.2, 0.0, big, big, None, 0, big, 256, 0))
topo = B.topology_build(B.RING, 8)
print(topo.n, topo.period)
"""


def _run(without):
    code = CALLS % (ROOT, without, without)
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    return done.stdout.split()


def test_the_binding_works_without_the_module():
    assert _run(True) == _run(False) == ["-1", "-1", "-5", "-8", "-2", "-6", "8", "1"]


def test_a_build_without_the_headers_of_python_leaves_the_module_out(monkeypatch, tmp_path, capsys):
    from paper_2104_11981_b200 import build
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_calls.so"))
    monkeypatch.setattr(build.sysconfig, "get_paths", lambda: {"include": str(tmp_path)})
    build._build_calls(True)
    assert os.listdir(tmp_path) == [] and "Python.h" in capsys.readouterr().err
    monkeypatch.undo()
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_calls.so"))
    build._build_calls(True)
    assert os.listdir(tmp_path) == ["_calls.so"]
