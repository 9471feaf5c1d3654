"""Refusals of the packed and paged entry points.  Arguments are checked before the handle's device is, so on a machine
without a GPU an accepted call ends with SAMKV_ERR_CUDA (6) and a refused one with its own code."""
import ctypes

import pytest
import torch

from paper_2508_11661_b200 import binding as B
from paper_2508_11661_b200 import build

INVALID, UNSUPPORTED, CUDA = 1, 2, 6


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


class Call:
    """Arguments of the three calls with host memory behind the pointers (nothing is launched on these paths)."""

    def __init__(self, T=10, Hq=8, Hkv=2, d=128, dtype=1, n_seq=2):
        self.buf = torch.zeros(1 << 20, dtype=torch.uint8)
        base = (self.buf.data_ptr() + 255) // 256 * 256
        self.base = base
        e = 2 if dtype == 1 else 4
        self.handle = ctypes.c_void_p(base)          # never looked into: the current device is asked for first
        self.packed = B.samkv_packed_t(Hq, Hkv, d, dtype, n_seq, T, 0, base)
        at = base + 4096
        self.r = {}
        for name, heads in (("Q", Hq), ("K", Hkv), ("V", Hkv), ("O", Hq), ("K_out", Hkv), ("V_out", Hkv)):
            self.r[name] = B.samkv_rows_t(at, heads * d, d)
            at += T * heads * d * e
        self.pages = B.samkv_pages_t(base + (1 << 18), base + (1 << 19), base, 16, 4, 3)      # pools of up to 64 KB
        self.rope = B.samkv_rope_t(d, 0, 10000.0, None)
        self.cache_len, self.positions, self.lse, self.scale = base, None, None, 0.0

    def prefill(self):
        r = self.r
        return B.lib().samkv_prefill(self.handle, self.packed, r["Q"], r["K"], r["V"], self.scale, r["O"], self.lse, None)

    def append(self, with_q=True, with_rows=True, with_pages=True, with_rope=True):
        r = self.r
        return B.lib().samkv_append(self.handle, self.packed, r["K"], r["V"], self.pages if with_pages else None,
                                    self.cache_len, self.rope if with_rope else None, self.positions,
                                    r["Q"] if with_q else None, r["O"] if with_q else None,
                                    r["K_out"] if with_rows else None, r["V_out"] if with_rows else None, None)

    def attn(self):
        return B.lib().samkv_paged_attn(self.handle, self.packed, self.pages, self.cache_len, self.r["Q"], self.scale, 1,
                                        self.r["O"], self.lse, None)


no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="an accepted call would be launched with host pointers")
ALL = ("prefill", "append", "attn")


@no_gpu
def test_good_arguments_get_past_the_checks():
    for dtype in (0, 1):
        for name in ALL:
            assert getattr(Call(dtype=dtype), name)() == CUDA
    c = Call()
    assert c.append(with_q=False) == CUDA and c.append(with_rows=False) == CUDA and c.append(with_rope=False) == CUDA
    assert c.append(with_pages=False) == CUDA
    c = Call(T=0)
    assert c.prefill() == CUDA                     # nothing to do, but the handle is still checked


@no_gpu
@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("field,value,status", [
    ("n_q_heads", 0, INVALID), ("n_q_heads", 7, INVALID), ("n_kv_heads", 0, INVALID), ("n_q_heads", 66, UNSUPPORTED),
    ("head_dim", 96, UNSUPPORTED), ("dtype", 2, UNSUPPORTED), ("n_seq", 0, INVALID), ("n_seq", 65537, UNSUPPORTED),
    ("n_tokens", -1, INVALID), ("max_seq_tokens", -1, INVALID), ("seq_offsets", None, INVALID)])
def test_bad_descriptions(name, field, value, status):
    c = Call()
    setattr(c.packed, field, value)
    assert getattr(c, name)() == status
    assert B.lib().samkv_packed_workspace_bytes(c.packed) == 0 or field == "seq_offsets"


@no_gpu
def test_null_pointers():
    for name in ALL:
        c = Call()
        c.handle = None
        assert getattr(c, name)() == INVALID
        c = Call()
        c.packed = None
        assert getattr(c, name)() == INVALID
    for call, operands in (("prefill", "QKVO"), ("append", "KV"), ("attn", "QO")):
        for x in operands:
            c = Call()
            c.r[x] = None
            assert getattr(c, call)() == INVALID, (call, x)
            c = Call()
            c.r[x].data = None
            assert getattr(c, call)() == INVALID, (call, x)
    for field in ("K", "V", "block_table"):
        for call in ("append", "attn"):
            c = Call()
            setattr(c.pages, field, None)
            assert getattr(c, call)() == INVALID
    c = Call()
    c.cache_len = None
    assert c.attn() == INVALID and c.append() == CUDA           # the append takes it as 0
    c = Call()
    c.r["O"] = None                                             # Q without Q_out
    assert c.append() == INVALID
    c = Call()
    c.r["V_out"] = None
    assert c.append() == INVALID
    assert Call().append(with_rows=False, with_pages=False) == INVALID
    assert B.lib().samkv_packed_workspace_bytes(None) == 0


@no_gpu
@pytest.mark.parametrize("call,operand", [("prefill", "Q"), ("prefill", "K"), ("prefill", "V"), ("prefill", "O"),
                                          ("append", "K"), ("append", "V"), ("append", "Q"), ("append", "K_out"),
                                          ("attn", "Q"), ("attn", "O")])
def test_strides_and_alignment(call, operand):
    def status(**kw):
        c = Call()
        r = c.r[operand]
        for k, v in kw.items():
            setattr(r, k, v)
        return getattr(c, call)()

    data = getattr(Call().r[operand], "data")
    assert status(data=data + 8) == INVALID
    assert status(token_stride=64) == INVALID and status(head_stride=64) == INVALID
    assert status(token_stride=0) == INVALID and status(head_stride=0) == INVALID and status(token_stride=-1024) == INVALID
    assert status(token_stride=1028) == INVALID and status(head_stride=132) == INVALID
    assert status(token_stride=1 << 37) == UNSUPPORTED


@no_gpu
def test_outputs_must_not_overlap():
    c = Call()
    c.r["O"].token_stride = 128                                  # rows of neighbouring tokens share memory
    assert c.prefill() == INVALID
    c = Call()
    c.r["O"] = c.r["Q"]
    assert c.prefill() == INVALID and c.attn() == INVALID
    assert c.append() == CUDA                                    # in place: the very rows of the input
    c.r["O"] = B.samkv_rows_t(c.r["Q"].data + 16, 1024, 128)
    assert c.append() == INVALID
    c = Call()
    c.r["V_out"] = c.r["K_out"]
    assert c.append() == INVALID
    c = Call()
    c.r["K_out"] = c.r["V"]                                      # K_out on V's rows
    assert c.append() == INVALID
    # slices of one fused matrix share an address range, not rows
    c = Call()
    w = (8 + 2 + 2) * 128
    base = c.base + 4096
    c.r["Q"], c.r["K"], c.r["V"] = (B.samkv_rows_t(base + 2 * off * 128, w, 128) for off in (0, 8, 10))
    c.r["O"] = c.r["Q"]
    c.r["K_out"], c.r["V_out"] = c.r["K"], c.r["V"]
    assert c.append() == CUDA and c.prefill() == INVALID
    c.r["O"] = B.samkv_rows_t(base + 2 * 10 * w, 8 * 128, 128)
    assert c.prefill() == CUDA


@no_gpu
def test_pools_must_not_overlap_what_a_call_reads_or_writes():
    pool = 4 * 2 * 16 * 128 * 2
    for which in ("K", "V"):
        def moved(**kw):
            c = Call()
            start = getattr(c.pages, which)
            for name, (back, rows_from_end) in kw.items():
                heads = 8 if name in ("Q", "O") else 2
                c.r[name] = B.samkv_rows_t(start + (pool if rows_from_end else -10 * heads * 128 * 2) + back, heads * 128, 128)
            return c

        for name in ("Q", "K", "V", "O", "K_out", "V_out"):
            assert moved(**{name: (0, True)}).append() == CUDA and moved(**{name: (0, False)}).append() == CUDA
            assert moved(**{name: (-16, True)}).append() == INVALID and moved(**{name: (16, False)}).append() == INVALID
        assert moved(O=(0, True)).attn() == CUDA and moved(O=(-16, True)).attn() == INVALID
        assert moved(Q=(-16, True)).attn() == CUDA            # both only read
    c = Call()
    c.pages.V = c.pages.K + pool - 16
    assert c.append() == INVALID and c.attn() == CUDA
    c.pages.V = c.pages.K + pool
    assert c.append() == CUDA


@no_gpu
def test_one_token_and_one_head_ignore_their_stride():
    c = Call(T=1)
    c.r["Q"].token_stride = 0
    assert c.prefill() == CUDA
    c = Call(Hq=2, Hkv=1)
    c.r["K"].head_stride = 0
    assert c.prefill() == CUDA


@no_gpu
@pytest.mark.parametrize("field,value,status", [
    ("page_size", 0, UNSUPPORTED), ("page_size", 8, UNSUPPORTED), ("page_size", 48, UNSUPPORTED), ("page_size", 512, UNSUPPORTED),
    ("page_size", -16, UNSUPPORTED), ("n_pages", 0, INVALID), ("table_width", 0, INVALID), ("table_width", 1 << 27, UNSUPPORTED),
    ("n_pages", 1 << 26, UNSUPPORTED)])
def test_bad_pages(field, value, status):
    for call in ("append", "attn"):
        c = Call()
        setattr(c.pages, field, value)
        assert getattr(c, call)() == status


@no_gpu
def test_bad_rotations_and_scales():
    def status(**kw):
        c = Call()
        for k, v in kw.items():
            setattr(c.rope, k, v)
        return c.append()

    assert status(rot_dim=0) == INVALID and status(rot_dim=24) == INVALID and status(rot_dim=144) == INVALID
    assert status(rot_dim=64) == CUDA
    for bad in (0.0, -1.0, float("inf"), float("nan")):
        assert status(base=bad) == INVALID
    freq = (ctypes.c_double * 64)(*([1.0] * 63 + [float("nan")]))
    assert status(inv_freq=ctypes.cast(freq, ctypes.POINTER(ctypes.c_double))) == INVALID
    freq[63] = 0.5
    assert status(inv_freq=ctypes.cast(freq, ctypes.POINTER(ctypes.c_double)), base=0.0) == CUDA
    c = Call()
    c.scale = float("nan")
    assert c.prefill() == INVALID and c.attn() == INVALID


def test_binding_checks_devices_types_and_shapes():
    off = torch.tensor([0, 3], dtype=torch.int32)
    with pytest.raises(ValueError):
        B.Packed(8, 2, 128, off.long(), 3)
    p = B.Packed(8, 2, 128, off, 3)
    assert p.n_seq == 1 and B.samkv_packed_workspace_bytes(p) >= 256
    with pytest.raises(ValueError):
        p.rows(torch.zeros(3, 8, 128, dtype=torch.bfloat16), (3, 8, 128), "Q", 0)          # host memory
    with pytest.raises(ValueError):
        B.Pages(torch.zeros(4, 2, 16, 128), torch.zeros(4, 2, 16, 64), off[None])
    with pytest.raises(ValueError):
        B.Pages(torch.zeros(4, 2, 16), torch.zeros(4, 2, 16, 128), off[None])
    with pytest.raises(ValueError):
        B.Rope(64, inv_freq=[1.0] * 31)
