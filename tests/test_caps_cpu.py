"""Numbers that describe modified scores: which caps a call takes, what the binding takes, and how good the bf16 kernels' polynomial is."""
import math
import os
import re
import sys

import numpy as np
import pytest

from paper_2508_11661_b200 import binding as B
from paper_2508_11661_b200 import build

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


def coefficients():
    with open(os.path.join(build.CSRC, "packed_cap.cuh")) as f:
        text = re.search(r"kTanh\[6\] = \{([^}]*)\}", f.read()).group(1)
    return np.array([float(x.strip().rstrip("f")) for x in text.split(",")], dtype=np.float32)


def test_the_polynomial_is_as_good_as_promised():
    """c tanh(x scale / c) log2(e) in the kernels' steps, every one rounded to fp32, against 64 bits: 2^-20 of the value.

    What adds up: the polynomial itself (checked first), then half a step, 2^-24 relative, for each of the factors in and out,
    the product y (its error reaches the result at most as it is: tanh's relative condition is <= 1), the scaled first
    coefficient, the last addition and the last product."""
    f, f8 = np.float32, np.float64
    k = coefficients()
    y = np.linspace(1e-4, 1, 100001)
    own = np.abs(y * np.polyval(k[::-1].astype(f8), y * y) / np.tanh(y) - 1).max()
    assert own < 2.0 ** -20.6
    rng = np.random.default_rng(0)
    y = np.concatenate([np.linspace(1e-3, 1, 6001), np.logspace(-6, 0, 1000)])
    for i in range(100):
        cap, scale = f(np.exp(rng.uniform(-8, 8))), f(rng.choice([0.125, 128 ** -0.5, 1.0, np.exp(rng.uniform(-3, 1))]))
        if i < 4:
            cap = f([1.5524435, 49.95557449, 50.0, 30.0][i])
        x = (y * f8(cap) / f8(scale)).astype(f)
        into, out = f(scale / cap), f(cap * f(math.log2(math.e)))
        c, at = (k * out).astype(f), (x * into).astype(f)
        z = (at * at).astype(f)
        q = np.full_like(z, c[5])
        for j in (4, 3, 2, 1, 0):
            q = (q.astype(f8) * z + f8(c[j])).astype(f)        # (one rounding: the product of two fp32 is exact in 64 bits)
        got = (at * q).astype(f8)
        want = f8(cap) * math.log2(math.e) * np.tanh(x.astype(f8) * f8(scale) / f8(cap))
        inside = np.abs(at) <= 1
        off = (np.abs(got - want) / want)[inside].max()
        assert off <= min(2.0 ** -20, own + 7 * 2.0 ** -24), (cap, scale, np.log2(off))
