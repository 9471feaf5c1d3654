"""Refusals of the page, multi-axis and modified-score entry points.  Arguments are checked before the handle's device is, so
on a machine without a GPU an accepted call ends with SAMKV_ERR_CUDA (6) and a refused one with its own code."""
import ctypes

import pytest
import torch

from paper_2508_11661_b200 import binding as B
from paper_2508_11661_b200 import build

INVALID, UNSUPPORTED, CUDA = 1, 2, 6
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="an accepted call would be launched with host pointers")


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


class Call:
    """Arguments of the calls with host memory behind the pointers (nothing is launched on these paths)."""

    def __init__(self, T=10, Hq=8, Hkv=2, d=128, dtype=1, n_seq=2):
        self.buf = torch.zeros(1 << 20, dtype=torch.uint8)
        base = (self.buf.data_ptr() + 255) // 256 * 256
        self.handle = ctypes.c_void_p(base)
        self.packed = B.samkv_packed_t(Hq, Hkv, d, dtype, n_seq, T, 0, base)
        e, at = 2 if dtype == 1 else 4, base + 4096
        self.r = {}
        for name, heads in (("Q", Hq), ("K", Hkv), ("V", Hkv), ("O", Hq), ("K_out", Hkv), ("V_out", Hkv)):
            self.r[name] = B.samkv_rows_t(at, heads * d, d)
            at += T * heads * d * e
        self.pages = B.samkv_pages_t(base + (1 << 18), base + (1 << 19), base, 16, 4, 3)
        self.a = {name: base + 65536 * 10 + 1024 * i for i, name in enumerate(
            ("cache_len", "table", "free", "n_free", "n_out", "slots", "positions", "total", "done", "slopes", "prefix", "doc"))}
        self.page_size, self.n_pages, self.width, self.n_seq = 16, 4, 3, n_seq
        self.axis = (ctypes.c_int32 * 64)(*[i % 3 for i in range(64)])
        self.rope = B.samkv_rope_axes_t(B.samkv_rope_t(d, 0, 10000.0, None), 3, ctypes.cast(self.axis, ctypes.POINTER(ctypes.c_int32)))
        self.stride = T
        self.scores = B.samkv_scores_t(30.0, 5, self.a["slopes"], self.a["prefix"], self.a["doc"])
        self.scale = 0.0

    def tables(self):
        a = self.a
        return B.lib().samkv_page_tables(self.handle, self.packed, a["cache_len"], self.page_size, self.n_pages, a["table"], self.width,
                                         a["free"], a["n_free"], a["n_out"], a["slots"], a["positions"], a["total"], None)

    def release(self):
        a = self.a
        return B.lib().samkv_release_pages(self.handle, self.n_seq, a["table"], self.width, self.page_size, self.n_pages,
                                           a["total"], a["done"], a["free"], a["n_free"], a["n_out"], None)

    def axes(self, with_rows=True, with_pages=True):
        r, a = self.r, self.a
        return B.lib().samkv_append_axes(self.handle, self.packed, r["K"], r["V"], self.pages if with_pages else None,
                                         a["cache_len"], a["slots"], self.rope, a["positions"], self.stride, r["Q"], r["O"],
                                         r["K_out"] if with_rows else None, r["V_out"] if with_rows else None, None)

    def prefill(self):
        r = self.r
        return B.lib().samkv_prefill_scores(self.handle, self.packed, r["Q"], r["K"], r["V"], self.scale, self.scores, r["O"], None, None)

    def attn(self):
        return B.lib().samkv_paged_attn_scores(self.handle, self.packed, self.pages, self.a["cache_len"], self.r["Q"], self.scale, 1,
                                               self.scores, self.r["O"], None, None)


def made(**kw):
    c = Call()
    for k, v in kw.items():
        if k in c.a:
            c.a[k] = v
        else:
            setattr(c, k, v)
    return c


ALL = ("tables", "release", "axes", "prefill", "attn")


@no_gpu
def test_good_arguments_get_past_the_checks():
    for dtype in (0, 1):
        for name in ALL:
            assert getattr(Call(dtype=dtype), name)() == CUDA
    assert Call().axes(with_rows=False) == CUDA
    assert made(slots=None).axes(with_pages=False) == CUDA
    assert made(rope=None, positions=None).axes() == CUDA and made(slots=None, positions=None).axes() == CUDA
    assert made(scores=None).prefill() == CUDA and made(scores=None).attn() == CUDA
    assert made(cache_len=None).tables() == CUDA
    assert made(slots=None, positions=None, total=None).tables() == CUDA
    for name in ALL:
        if name != "release":
            assert getattr(Call(T=0), name)() == CUDA
    c = Call()
    c.a["n_out"] = c.a["n_free"]
    assert c.tables() == CUDA and c.release() == CUDA


@no_gpu
@pytest.mark.parametrize("name", ["tables", "axes", "prefill", "attn"])
@pytest.mark.parametrize("field,value,status", [
    ("n_q_heads", 7, INVALID), ("n_q_heads", 66, UNSUPPORTED), ("head_dim", 96, UNSUPPORTED), ("dtype", 2, UNSUPPORTED),
    ("n_seq", 0, INVALID), ("n_seq", 65537, UNSUPPORTED), ("n_tokens", -1, INVALID), ("seq_offsets", None, INVALID)])
def test_bad_descriptions(name, field, value, status):
    c = Call()
    setattr(c.packed, field, value)
    assert getattr(c, name)() == status
    assert B.lib().samkv_scores_workspace_bytes(c.packed) == 0 or field == "seq_offsets"


@no_gpu
def test_null_and_misaligned_pointers():
    for name in ALL:
        c = Call()
        c.handle = None
        assert getattr(c, name)() == INVALID
        if name != "release":
            assert getattr(made(packed=None), name)() == INVALID
    for field in ("table", "free", "n_free", "n_out"):
        assert made(**{field: None}).tables() == INVALID and made(**{field: None}).release() == INVALID
    for field in ("total", "done"):
        assert made(**{field: None}).release() == INVALID
    for field in ("cache_len", "table", "free", "n_free", "n_out", "slots", "positions", "total"):
        assert made(**{field: Call().a[field] + 2}).tables() == INVALID
    assert made(cache_len=None).attn() == INVALID
    assert made(slots=Call().a["slots"] + 2).axes() == INVALID and made(positions=Call().a["positions"] + 1).axes() == INVALID
    for field in ("slopes", "prefix_len", "doc_start"):
        c = Call()
        setattr(c.scores, field, getattr(c.scores, field) + 2)
        assert c.prefill() == INVALID and c.attn() == INVALID


@no_gpu
@pytest.mark.parametrize("field,value,status", [
    ("page_size", 8, UNSUPPORTED), ("page_size", 48, UNSUPPORTED), ("page_size", 0, UNSUPPORTED), ("n_pages", 0, INVALID),
    ("width", 0, INVALID), ("width", 1 << 27, UNSUPPORTED), ("n_pages", 1 << 28, UNSUPPORTED)])
def test_bad_pages(field, value, status):
    assert made(**{field: value}).tables() == status and made(**{field: value}).release() == status


@no_gpu
def test_page_arrays_must_not_overlap():
    names = ("cache_len", "free", "n_free", "table", "n_out", "slots", "positions", "total")
    outs = ("table", "n_out", "slots", "positions", "total")
    for i in names:
        for j in outs:
            c = Call()
            if i != j:
                c.a[j] = c.a[i]
                assert c.tables() == (CUDA if {i, j} == {"n_free", "n_out"} else INVALID), (i, j)
    c = Call()
    c.a["total"] = c.a["cache_len"] + 4
    assert c.tables() == INVALID
    c.a["total"] = c.a["cache_len"] + 8
    assert c.tables() == CUDA
    for i in ("table", "total", "done", "n_free"):
        for j in ("free", "n_out"):
            c = Call()
            c.a[j] = c.a[i]
            assert c.release() == (CUDA if (i, j) == ("n_free", "n_out") else INVALID), (i, j)
    assert made(n_seq=0).release() == INVALID and made(n_seq=65537).release() == UNSUPPORTED


@no_gpu
def test_bad_axes():
    def status(**kw):
        c = Call()
        for k, v in kw.items():
            setattr(c.rope, k, v)
        return c.axes()

    assert status(n_axes=0) == INVALID and status(n_axes=5) == INVALID and status(n_axes=2) == INVALID
    assert status(n_axes=4) == CUDA
    assert status(pair_axis=None) == INVALID
    c = Call()
    c.axis[63] = -1
    assert c.axes() == INVALID
    for rot in (0, 24, 144, 8, -16):
        c = Call()
        c.rope.rope.rot_dim = rot
        assert c.axes() == INVALID
    c = Call()
    c.rope.rope.base = -1.0
    assert c.axes() == INVALID
    assert made(stride=9).axes() == INVALID and made(stride=-1).axes() == INVALID and made(stride=0).axes() == CUDA
    assert made(stride=1 << 41).axes() == UNSUPPORTED
    assert made(positions=None).axes() == INVALID                 # the slot map does not say where a token stands
    assert Call().axes(with_pages=False) == INVALID


@no_gpu
def test_bad_scores():
    def status(scale=0.0, **kw):
        c = Call()
        c.scale = scale
        for k, v in kw.items():
            setattr(c.scores, k, v)
        assert c.prefill() == c.attn()
        return c.prefill()

    for bad in (-1.0, float("nan"), float("inf"), 1e31, 1e-42):
        assert status(softcap=bad) == INVALID
    assert status(softcap=1e-38, scale=1e3) == INVALID and status(softcap=1e-3) == CUDA and status(softcap=0.0) == CUDA
    assert status(window=-1) == INVALID and status(window=2 ** 31 - 1) == CUDA
    assert status(scale=float("nan")) == INVALID


@no_gpu
def test_rows_and_overlaps_are_checked_as_in_the_plain_calls():
    for name in ("prefill", "attn", "axes"):
        for operand in ("Q", "O") if name != "axes" else ("Q", "K", "O", "K_out"):
            c = Call()
            c.r[operand].data += 8
            assert getattr(c, name)() == INVALID
            c = Call()
            c.r[operand].token_stride = 64
            assert getattr(c, name)() == INVALID
    c = Call()
    c.r["O"] = c.r["Q"]
    assert c.prefill() == INVALID and c.attn() == INVALID and c.axes() == CUDA


def test_workspace_serves_the_plain_calls_too():
    for dtype in (0, 1):
        for T, n_seq in ((0, 1), (10, 2), (100000, 3), (5000, 65536)):
            p = B.samkv_packed_t(8, 2, 128, dtype, n_seq, T, 0, None)
            assert B.lib().samkv_scores_workspace_bytes(p) >= B.lib().samkv_packed_workspace_bytes(p) > 0
    assert B.lib().samkv_scores_workspace_bytes(None) == 0


def test_binding_checks_types_and_shapes():
    i32 = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.Scores(slopes=torch.zeros(3, dtype=torch.float64))
    with pytest.raises(ValueError):
        B.Scores(prefix_len=i32.long())
    with pytest.raises(ValueError):
        B.Scores(doc_start=torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.RopeAxes(64, [0] * 31)
    r = B.RopeAxes.sections([2, 3, 3])
    assert r.n_axes == 3 and r.c.rope.rot_dim == 16 and [r.c.pair_axis[i] for i in range(8)] == [0, 0, 1, 1, 1, 2, 2, 2]
