"""The extension module of the binding is an extra: the library is built and used without it, and with one that was built for
another Python or torch."""
import os
import subprocess
import sys
import sysconfig

import pytest
import torch

from paper_2508_11661_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(autouse=True)
def elsewhere(tmp_path, monkeypatch):
    """The module of these tests lies in a folder of its own."""
    build.build_library()
    monkeypatch.setattr(build, "MARSHAL_PATH", str(tmp_path / os.path.basename(build.MARSHAL_PATH)))
    return tmp_path


def fake_compiler(monkeypatch, status):
    """Commands that are asked for, instead of running them; g++ writes its output or fails."""
    asked = []

    def check_call(cmd, **kw):
        asked.append(cmd)
        out = cmd[cmd.index("-o") + 1]
        with open(out, "wb") as f:
            f.write(b"half")
        if status:
            raise status
    monkeypatch.setattr(build.subprocess, "check_call", check_call)
    return asked


@pytest.mark.parametrize("status", [subprocess.CalledProcessError(1, "g++"), FileNotFoundError("g++")])
def test_the_library_is_built_without_a_host_compiler(monkeypatch, elsewhere, status):
    asked = fake_compiler(monkeypatch, status)
    with pytest.warns(RuntimeWarning, match="_marshal"):
        assert build.build_library() == build.LIB_PATH
    assert len(asked) == 1 and not os.path.exists(build.MARSHAL_PATH)
    assert os.listdir(elsewhere) == []                   # nothing half written stays


def test_a_module_that_cannot_be_rebuilt_does_not_stay(monkeypatch):
    with open(build.MARSHAL_PATH, "wb") as f:
        f.write(b"old")
    os.utime(build.MARSHAL_PATH, (1, 1))
    fake_compiler(monkeypatch, subprocess.CalledProcessError(1, "g++"))
    with pytest.warns(RuntimeWarning, match="_marshal"):
        build.build_library()
    assert not os.path.exists(build.MARSHAL_PATH)


def test_the_module_is_built_again_for_another_torch(monkeypatch):
    asked = fake_compiler(monkeypatch, None)
    assert build.build_marshal() == build.MARSHAL_PATH and len(asked) == 1
    assert build.build_marshal() == build.MARSHAL_PATH and len(asked) == 1
    assert os.path.exists(build.MARSHAL_PATH)
    monkeypatch.setattr(torch, "__version__", "99.0")
    build.build_marshal()
    assert len(asked) == 2 and any("99.0" in a for a in asked[1])
    build.build_marshal()
    assert len(asked) == 2
    build.build_marshal(force=True)
    assert len(asked) == 3
    os.utime(build.MARSHAL_PATH, (1, 1))                 # older than its sources
    build.build_marshal()
    assert len(asked) == 4


def test_the_name_says_for_which_python():
    assert os.path.basename(build.MARSHAL_PATH) == "_marshal" + sysconfig.get_config_var("EXT_SUFFIX")


@pytest.mark.parametrize("version,used", [("torch.__version__", True), ("'0.1'", False), (None, False)])
def test_a_module_for_another_torch_is_not_used(version, used):
    code = f"""
import sys, types
import torch
m = types.ModuleType("paper_2508_11661_b200._marshal")
{'m.torch_version = ' + version if version else ''}
m.otherwise, m.device_ptr, m.rows = lambda *a: None, len, len
sys.modules[m.__name__] = m
from paper_2508_11661_b200 import binding as B
assert (B._rows is len) == {used}, B._rows
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]


def test_the_built_module_is_for_this_torch():
    from paper_2508_11661_b200 import _marshal
    assert _marshal.torch_version == torch.__version__
