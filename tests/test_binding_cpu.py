"""The packed calls' way through the binding, on host tensors: with the extension module and with the Python forms that stand
in for it.  Everything runs in a process of its own, since what is wrong with an argument must not end the caller's."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2508_11661_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="an accepted call would be launched with host pointers")

# Host tensors have device -1; with that as the current device a call goes all the way to the library, which answers
# SAMKV_ERR_CUDA (6) where it accepts the arguments and there is no GPU.
SETUP = """
import ctypes, sys, types
import numpy as np
import torch
MODULE = {module}
if not MODULE:
    sys.modules["paper_2508_11661_b200._marshal"] = None
from paper_2508_11661_b200 import binding as B
assert (getattr(B, "_marshal", None) is not None) == MODULE
B._current_device, B._raw_stream = lambda: -1, lambda device: 0

def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)

memory = torch.zeros(1 << 16, dtype=torch.uint8)
handle = types.SimpleNamespace(_h=ctypes.c_void_p((memory.data_ptr() + 255) // 256 * 256))
T, Hq, Hkv, d = 10, 8, 2, 64
offsets = torch.tensor([0, 4, 10], dtype=torch.int32)
packed = B.Packed(Hq, Hkv, d, offsets, T, dtype="f32")
Q, K, V, O = torch.zeros(T, Hq, d), torch.zeros(T, Hkv, d), torch.zeros(T, Hkv, d), torch.zeros(T, Hq, d)
lse = torch.zeros(T, Hq)

def outcome(f, *args, **kw):
    try:
        f(*args, **kw)
        return "OK"
    except B.SamkvError as e:
        return str(e).split(": ")[1].split(" ")[0]
    except Exception as e:
        return type(e).__name__
"""


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


def run(code, module):
    r = subprocess.run([sys.executable, "-c", SETUP.format(module=module) + code], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]


both = pytest.mark.parametrize("module", [True, False], ids=["module", "python"])


@no_gpu
@both
def test_tensors_without_memory_raise(module):
    """Tensors inside torch.vmap and torch.func.grad, and fake ones, have a type, a shape and a device but no address."""
    run("""
assert outcome(B.samkv_prefill, handle, packed, Q, K, V, 0.0, O, lse) == "SAMKV_ERR_CUDA"
seen = []
def rows(x):
    seen.append(outcome(B.samkv_prefill, handle, packed, x, K, V, 0.0, O, lse))
    return x
def plain(x):
    seen.append(outcome(B.samkv_prefill, handle, packed, Q, K, V, 0.0, O, x))
    return x.sum()
torch.vmap(rows)(torch.zeros(3, T, Hq, d))
torch.vmap(plain)(torch.zeros(3, T, Hq))
torch.func.grad(plain)(torch.zeros(T, Hq))
assert seen == ["RuntimeError"] * 3, seen
from torch._subclasses.fake_tensor import FakeTensorMode
with FakeTensorMode():
    fake = torch.zeros(T, Hq, d)
assert outcome(B.samkv_prefill, handle, packed, fake, K, V, 0.0, O, lse) not in ("OK", "SAMKV_ERR_CUDA")
""", module)
