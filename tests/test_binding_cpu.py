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


@no_gpu
@both
def test_arguments_of_other_types(module):
    """A number that is no integer, or nothing that could be meant, is refused before the library sees any argument."""
    run("""
free, n_free, n_out, table = i32(16), i32(1), i32(1), i32(2, 3)
lengths, done = i32(2), torch.zeros(2, dtype=torch.bool)
def tables(page_size, scale=0.0):
    return outcome(B.samkv_page_tables, handle, packed, None, page_size, table, free, n_free, n_out)
def release(page_size):
    return outcome(B.samkv_release_pages, handle, table, page_size, lengths, done, free, n_free, n_out)
for f in (tables, release):
    for good in (16, np.int64(16), np.int32(16)):
        assert f(good) == "SAMKV_ERR_CUDA" or (not MODULE and type(good) is not int), (f, good)
    assert f(17) == "SAMKV_ERR_UNSUPPORTED"
    for bad in (16.0, np.float32(16.0), 2.5, "16", b"16", (16, 0, 0), packed.c, [16], 16j):
        assert f(bad) in ("TypeError", "ArgumentError"), (f, bad, f(bad))
assert outcome(B.samkv_prefill, handle, packed, Q, K, V, 1, O) == "SAMKV_ERR_CUDA"           # scale: any real number
assert outcome(B.samkv_prefill, handle, packed, Q, K, V, "1", O) in ("ValueError", "TypeError", "SAMKV_ERR_CUDA")
assert outcome(B.samkv_prefill, handle, packed, Q, K, V, [1], O) == "TypeError"
""", module)


def test_every_argument_arrives_in_its_place():
    """Each packed call of the extension module against a function that writes down what it gets."""
    run("""
NAMES = [n for n in dir(B._marshal) if n.startswith("samkv_")]
assert set(NAMES) == {n for n in B.EXPORTS if n in (
    "samkv_prefill", "samkv_append", "samkv_paged_attn", "samkv_page_tables", "samkv_release_pages", "samkv_append_axes",
    "samkv_prefill_scores", "samkv_paged_attn_scores")}, NAMES
for name in NAMES:
    types = getattr(B.lib(), name).argtypes
    got = []
    def note(*args):
        got[:] = [a if not isinstance(a, ctypes._Pointer) else bytes(a.contents) if a else None for a in args]
        return 5
    callback = ctypes.CFUNCTYPE(ctypes.c_int, *types)(note)
    address, call = ctypes.cast(callback, ctypes.c_void_p).value, getattr(B._marshal, name)
    args, want = [], []
    for i, t in enumerate(types):
        if t is ctypes.c_float:
            args.append(0.5 + i)
            want.append(0.5 + i)
        elif t is ctypes.POINTER(B.samkv_rows_t):
            args.append((4096 + i, 100 + i, 200 + i))
            want.append(bytes(B.samkv_rows_t(*args[-1])))
        elif hasattr(t, "contents"):
            s = t._type_()
            ctypes.memset(ctypes.byref(s), i + 1, ctypes.sizeof(s))
            args.append(s)
            want.append(bytes(s))
        elif t is ctypes.c_void_p:
            args.append((1 << 40) + i)
            want.append((1 << 40) + i)
        else:
            args.append((1 << 35) + i if t is ctypes.c_int64 else -1000 - i)
            want.append(args[-1])
    assert call(address, *args) == 5 and got == want, (name, got, want)
    # None is a null pointer, and nothing else
    for i, t in enumerate(types):
        now = list(args)
        now[i] = None
        if t in (ctypes.c_float, ctypes.c_int32, ctypes.c_int64):
            assert outcome(call, address, *now) == "TypeError", (name, i)
        else:
            assert call(address, *now) == 5 and got == want[:i] + [None] + want[i + 1:], (name, i)
        # what belongs elsewhere
        for bad in (2.5, 7, (1, 2, 3), (1, 2), b"x", memory.numpy(), ctypes.c_int32(3), "3"):
            now[i] = bad
            fits = (t is ctypes.c_float and type(bad) is float) or (t is ctypes.POINTER(B.samkv_rows_t) and bad == (1, 2, 3)) if not hasattr(bad, "shape") else False
            fits = fits or (type(bad) is int and t in (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64))
            assert (outcome(call, address, *now) == "OK") == fits, (name, i, t, bad)
    for wrong in (args[:-1], args + [0], []):
        assert outcome(call, address, *wrong) == "TypeError"
    assert outcome(call) == "TypeError" and outcome(call, 1.0, *args) == "TypeError" and outcome(call, 0, *args) == "TypeError"
    for i, t in enumerate(types):
        if t is ctypes.c_int32:
            assert outcome(call, address, *args[:i], 1 << 32, *args[i + 1:]) == "OverflowError"
""", True)
