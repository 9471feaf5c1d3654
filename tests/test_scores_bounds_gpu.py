"""Modified scores: the bounds of their parameters, rows beside one another, pages in the midst of a row tile."""
import pytest

from scores_testlib import Mods
from packed_testlib import PagedCase
from test_scores_gpu import check_paged, check_prompt, paged, prompt, randn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [2.0 ** -126, 1e30])
def test_smallest_and_largest_cap(dtype, cap):
    """Scores of exactly 0 among others; the smallest cap makes all of them one, the largest none of them another."""
    n = 150
    q, k, v = (randn(n, 2, 64, dtype=dtype, seed=i + 200) for i in range(3))
    q[5::7] = 0
    k[3::5] = 0
    mods = Mods(softcap=cap)
    O, lse = prompt(q, k, v, [n], dtype, mods)
    check_prompt(q, k, v, [n], dtype, mods, O, lse)
    c = PagedCase([1, 1], [130, 7], 4, 2, 64, 16, dtype, seed=201)
    c.Q[0] = 0
    O, lse = paged(c, mods, max_seq=1)
    check_paged(c, mods, O, lse)
