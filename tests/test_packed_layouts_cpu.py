"""Layouts of packed tensors that lie between one another without sharing a row, and ones that do share rows.  On a machine
without a GPU an accepted call ends with SAMKV_ERR_CUDA (6), see test_packed_cpu."""
import itertools

import numpy as np
import pytest
import torch

from paper_2508_11661_b200 import binding as B
from paper_2508_11661_b200 import build
from test_packed_cpu import CUDA, INVALID, Call, no_gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


@no_gpu
@pytest.mark.parametrize("T", [1, 10])
def test_heads_of_one_slab_may_alternate(T):
    """K and V of a document as [heads, 2, tokens, d]: their address ranges interleave, their rows do not."""
    c = Call(T=T)
    slab = c.base + 65536
    c.r["K_out"] = B.samkv_rows_t(slab, 128, 2 * T * 128)
    c.r["V_out"] = B.samkv_rows_t(slab + T * 256, 128, 2 * T * 128)
    assert c.append() == CUDA
    c.r["V_out"] = B.samkv_rows_t(slab + (T - 1) * 256 + 240, 128, 2 * T * 128)      # 16 bytes into the last row of K
    assert c.append() == INVALID
    c.r["V_out"] = B.samkv_rows_t(slab + T * 256 + 16, 128, 2 * T * 128)             # and 16 bytes into the next head's first
    assert c.append() == INVALID


@no_gpu
def test_overlap_agrees_with_a_count_of_the_bytes():
    """Accepted: no byte is shared.  (Refusing more than that is allowed, but not the layouts named above.)"""
    d, T = 64, 3
    layouts = [(128, 64), (192, 64), (64, 192), (64, 384), (256, 64), (320, 128), (128, 384)]

    def touched(start, ts, hs, heads):
        at = start + 2 * (np.arange(T)[:, None, None] * ts + np.arange(heads)[None, :, None] * hs + np.arange(d)[None, None, :])
        return set(at.reshape(-1).tolist())

    accepted = 0
    for (ts1, hs1), (ts2, hs2), shift in itertools.product(layouts, layouts, range(-512, 2049, 128)):
        c = Call(T=T, Hq=2, Hkv=2, d=d)
        at = c.base + 131072
        c.r["K_out"], c.r["V_out"] = B.samkv_rows_t(at, ts1, hs1), B.samkv_rows_t(at + shift, ts2, hs2)
        status = c.append(with_pages=False)
        assert status in (CUDA, INVALID)
        if status == CUDA:
            accepted += 1
            assert not touched(at, ts1, hs1, 2) & touched(at + shift, ts2, hs2, 2), (ts1, hs1, ts2, hs2, shift)
    assert accepted > 100
