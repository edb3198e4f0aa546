"""The C module of the calls is built beside any installation of the tensors, without their exchange interface where the header lacks it."""
import os
import types

import pytest

# what a header before the interface has
OLD = """
#define DLPACK_MAJOR_VERSION 1
typedef enum { kDLCPU = 1, kDLCUDA = 2 } DLDeviceType;
typedef struct { DLDeviceType device_type; int device_id; } DLDevice;
"""
# a draft of it, under another name
DRAFT = OLD + "typedef struct DLPackPyObjectExchangeAPI { int version; } DLPackPyObjectExchangeAPI;\n"


@pytest.mark.parametrize("header,has", [(None, False), (OLD, False), (DRAFT, False), ("installed", True)],
                         ids=["missing", "old", "draft", "installed"])
def test_the_module_is_built_with_any_header(header, has, monkeypatch, tmp_path):
    from paper_2104_11981_b200 import build
    if header != "installed":
        os.makedirs(tmp_path / "include" / "ATen")
        if header is not None:
            (tmp_path / "include" / "ATen" / "dlpack.h").write_text(header)
        spec = types.SimpleNamespace(origin=str(tmp_path / "__init__.py"))
        monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: spec)
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_calls.so"))
    build._build_calls(True)
    module = (tmp_path / "_calls.so").read_bytes()
    assert b"PyInit__calls" in module and (b"read_tensors" in module) == has
