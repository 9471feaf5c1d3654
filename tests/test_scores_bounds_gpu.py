"""Modified scores: the bounds of their parameters, rows beside one another, pages in the midst of a row tile."""
import numpy as np
import pytest
import torch

from paper_2508_11661_b200 import binding as B
from scores_testlib import Mods, attend64, check
from packed_testlib import PagedCase, f64
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


# tokens that see nothing in the midst of a row tile, or at its end
GONE = {
    # the first token sees what is before it, the last one itself: the pages of those between are nobody's
    "midst": (64, 32, lambda n, c: [0] + [1 << 29] * (n - 2) + [c + n - 1]),
    # only the first token sees anything: the pages behind its own are nobody's
    "end": (40, 31, lambda n, c: [0] + [1 << 29] * (n - 1)),
    "end of two": (2, 31, lambda n, c: [0, 1 << 29]),
    # nobody sees anything but the prefix
    "all": (40, 100, lambda n, c: [1 << 29] * n),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("where", list(GONE))
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (8, 2), (16, 1)])
def test_pages_that_no_token_sees_may_be_gone(dtype, where, Hq, Hkv):
    """Whatever the tokens around them see, and however the call's row tiles lie."""
    n, cached, starts = GONE[where]
    page = 16
    c = PagedCase([n, 3], [cached, 5], Hq, Hkv, 64, page, dtype, seed=210)
    mods = Mods(softcap=9.0, doc=np.array(starts(n, cached) + [0, 1, 2]), prefix=[3, 0])
    O, lse = paged(c, mods)
    check_paged(c, mods, O, lse)
    seen = mods.seen(0, 0, cached, n, cached + n).any(axis=0)
    gone = [col for col in range(-(-(cached + n) // page)) if not seen[col * page:(col + 1) * page].any()]
    assert gone
    for i, col in enumerate(gone):
        c.Kp[int(c.table[0, col])] = float("nan")
        c.Vp[int(c.table[0, col])] = float("inf")
        c.table[0, col] = [-1, 1 << 30, -(1 << 31)][i % 3]
    for max_seq in (0, n):
        O2, lse2 = paged(c, mods, max_seq=max_seq)        # (asks the device check word)
        check_paged(c, mods, O2, lse2)
    # one that a token does see is still recorded
    col = int(np.flatnonzero(seen)[-1]) // page
    c.table[0, col] = 1 << 30
    p = B.Packed(Hq, Hkv, 64, c.offsets, c.T, 0, dtype)
    h = B.Handle.for_scores(p)
    B.samkv_paged_attn_scores(h, p, B.Pages(c.Kp, c.Vp, c.table), c.cache_len, c.Q, 0.0, True, mods.device(B, DEV), torch.empty_like(c.Q))
    assert B.samkv_poll_status(h) == 7


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("softcap", [0.0, 3.0])
def test_a_token_does_not_depend_on_those_beside_it(dtype, softcap):
    """The token at position 63 as the last of a chunk and as the first of one: the same bits."""
    Hq, d, n = 8, 64, 32
    slopes = np.random.default_rng(11).uniform(0.01, 0.3, Hq)
    results = []
    pools = PagedCase([n], [63], Hq, Hq, d, 16, dtype, seed=220)
    token = randn(1, Hq, d, dtype=dtype, seed=221, gain=3.0)
    for cached, row in ((32, 31), (63, 0), (50, 13)):
        c = PagedCase([n], [cached], Hq, Hq, d, 16, dtype, seed=222)
        c.Kp, c.Vp, c.table, c.n_pages = pools.Kp, pools.Vp, pools.table, pools.n_pages
        c.Q[row] = token[0]
        O, lse = paged(c, Mods(softcap=softcap, slopes=slopes))
        results.append((O[row], lse[row]))
    for O, lse in results[1:]:
        assert torch.equal(O, results[0][0]) and torch.equal(lse, results[0][1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [0, 70])
def test_causal_instruction_documents_and_question(dtype, window):
    """A causal model's instruction goes first, by a call without a prefix; documents that do not see one another and a question
    that sees all follow as a chunk behind it, with the instruction as their prefix.  (With a window: initial tokens kept.)"""
    pre, n, doc_len, tail, Hq, Hkv, d = 45, 400, 150, 30, 8, 2, 64
    first = PagedCase([pre], [0], Hq, Hkv, d, 16, dtype, seed=230)
    rest = PagedCase([n], [pre], Hq, Hkv, d, 16, dtype, seed=231)
    first.Kp, first.Vp, first.table, first.table_cpu, first.n_pages = rest.Kp, rest.Vp, rest.table, rest.table_cpu, rest.n_pages
    t = np.arange(n)
    doc = np.zeros(n, dtype=np.int64) if window else np.where(t < n - tail, pre + t // doc_len * doc_len, 0)
    mods = Mods(window=window, prefix=[pre], doc=doc)
    O1, lse1 = paged(first, Mods(window=window))
    O2, lse2 = paged(rest, mods)
    # the model: every token of the one sequence sees what is at or before it, of the instruction or of its own document
    p, j = np.arange(pre + n)[:, None], np.arange(pre + n)[None, :]
    start = np.concatenate([np.zeros(pre, dtype=np.int64), doc])[:, None]
    ok = (j <= p) & ((j < pre) | ((j >= start) & ((p - j < window) if window else True)))
    q = np.concatenate([f64(first.Q), f64(rest.Q)])
    ref = attend64(q, rest.slots(rest.Kp, 0, pre + n), rest.slots(rest.Vp, 0, pre + n), ok, np.arange(pre + n), mods, d ** -0.5)
    check(np.concatenate([f64(O1), f64(O2)]), np.concatenate([f64(lse1), f64(lse2)]), ref, dtype, pre + n)
    # in one call the instruction's tokens see one another in both directions
    both = PagedCase([pre + n], [0], Hq, Hkv, d, 16, dtype, seed=231)
    both.Kp, both.Vp, both.table, both.n_pages = rest.Kp, rest.Vp, rest.table, rest.n_pages
    both.Q = torch.cat([first.Q, rest.Q])
    O, lse = paged(both, Mods(window=window, prefix=[pre], doc=np.concatenate([np.zeros(pre, dtype=np.int64), doc])))
    ok[:pre, :pre] = True
    ref = attend64(q, rest.slots(rest.Kp, 0, pre + n), rest.slots(rest.Vp, 0, pre + n), ok, np.arange(pre + n), mods, d ** -0.5)
    check(f64(O), f64(lse), ref, dtype, pre + n)
