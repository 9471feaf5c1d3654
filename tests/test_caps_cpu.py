"""Which caps a call with modified scores takes, and how good the bf16 kernels' polynomial is."""
import os
import sys

import pytest

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
