"""Numbers that describe modified scores: which caps a call takes, what the binding takes, and how good the bf16 kernels' polynomial is."""
import os
import sys

import numpy as np
import pytest

from paper_2508_11661_b200 import binding as B

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_scores_cpu import CUDA, INVALID, Call, _built, no_gpu  # noqa: E402,F401

SMALLEST, LARGEST = 2.0 ** -126, 1e30


@no_gpu
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("softcap,scale,status", [
    # the reciprocal of a cap below 2^-126 may be no fp32 number
    (2e-39, 0.0, INVALID), (3.7e-40, 0.0, INVALID), (2.9e-39, 0.0, INVALID), (1.17549e-38, 0.0, INVALID), (1e-45, 1e-30, INVALID),
    (SMALLEST, 0.0, CUDA), (SMALLEST, 1.0, CUDA), (SMALLEST, 5.0, INVALID), (LARGEST, 0.0, CUDA), (1.001e30, 0.0, INVALID),
    (LARGEST, 1e-9, CUDA), (50.0, 5e-37, CUDA), (30.0, float("inf"), INVALID)])
def test_bounds_of_caps(dtype, softcap, scale, status):
    c = Call(dtype=dtype)
    c.scores.softcap, c.scale = softcap, scale
    assert c.prefill() == status and c.attn() == status


def test_numbers_that_do_not_fit_are_refused():
    """A cap that fp32 rounds to 0 would be no cap, a window of 2^32 no window."""
    for kw in (dict(softcap=1e-46), dict(softcap=1e39), dict(softcap=-1e-50), dict(window=1 << 32), dict(window=(1 << 32) + 5),
               dict(window=1 << 31), dict(window=(-1 << 31) - 1)):
        with pytest.raises((ValueError, OverflowError)):
            B.Scores(**kw)
    for kw in (dict(window=3.0), dict(window="3"), dict(softcap="5")):
        with pytest.raises(TypeError):
            B.Scores(**kw)
    s = B.Scores(softcap=np.float32(2.0), window=np.int64(7))
    assert s.c.softcap == 2.0 and s.c.window == 7
    assert B.Scores(softcap=0).c.softcap == 0.0 and B.Scores(window=2 ** 31 - 1).c.window == 2 ** 31 - 1
    for axes in ([1 << 32] * 8, [0] * 7 + [(1 << 32) + 1], [-1 << 32] + [0] * 7):
        with pytest.raises((ValueError, OverflowError)):
            B.RopeAxes(16, axes)
