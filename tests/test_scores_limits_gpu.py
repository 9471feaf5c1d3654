"""Modified scores and pages at their limits: long caches in waves, captured calls with a plan of their own, two handles at once,
small workspaces."""
import numpy as np
import pytest
import torch

from paper_2508_11661_b200 import binding as B
from packed_testlib import DT, PagedCase, f64
from scores_testlib import Mods, attend64, check
from test_scores_gpu import check_paged, check_prompt, mods_of, offsets_of, paged, prompt, randn, slopes_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("kind", ["cap", "slope", "cap+slope+prefix", "doc"])
@pytest.mark.parametrize("new,cached", [([128], [140000]), ([100, 27], [9000, 150001])])
def test_row_tiles_that_share_a_long_cache(kind, new, cached):
    """Several row tiles over more keys than half the L2 cache holds: blocks of the cache run in waves."""
    Hq, Hkv, d = 16, 2, 64
    c = PagedCase(new, cached, Hq, Hkv, d, 256, "bf16", seed=200)
    c.Q *= 3
    mods = mods_of(kind, new, cached, Hq, seed=9)
    if mods.slopes is not None:
        mods.slopes = mods.slopes * 1e-3                      # (far slots count)
    O, lse = paged(c, mods)
    check_paged(c, mods, O, lse, sample=[0, 15, 16, 26, 99, 127])
    again, lse2 = paged(c, mods)
    assert torch.equal(O, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_replay_of_calls_with_a_plan_kernel(dtype):
    """More row tiles than a warp plans by itself, captured once and replayed with other lengths and masks."""
    T, n_seq, Hq, Hkv, d = 900, 60, 8, 2, 64
    q, k, v = (randn(T, h, d, dtype=dtype, seed=i + 210) for i, h in enumerate((Hq, Hkv, Hkv)))
    offsets = torch.zeros(n_seq + 1, dtype=torch.int32, device=DEV)
    p = B.Packed(Hq, Hkv, d, offsets, T, 0, dtype)
    h = B.Handle.for_scores(p)
    scores = B.Scores(softcap=5.0, window=150, slopes=torch.zeros(Hq, device=DEV), prefix_len=torch.zeros(n_seq, dtype=torch.int32, device=DEV),
                      doc_start=torch.zeros(T, dtype=torch.int32, device=DEV))
    O, lse = torch.zeros_like(q), torch.zeros((T, Hq), device=DEV)

    def call():
        B.samkv_prefill_scores(h, p, q, k, v, 0.0, scores, O, lse)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    r = np.random.default_rng(3)
    for new in ([15] * 60, [900] + [0] * 59, [0, 1, 500, 0, 300] + [1] * 55, [0] * 59 + [7]):
        mods = Mods(softcap=5.0, window=150, slopes=slopes_of(Hq) * r.random(), prefix=r.integers(0, 40, n_seq), doc=r.integers(-3, 200, T))
        offsets.copy_(offsets_of(new))
        scores.slopes.copy_(torch.from_numpy(mods.slopes))
        scores.prefix_len.copy_(torch.tensor(mods.prefix, dtype=torch.int32))
        scores.doc_start.copy_(torch.tensor(mods.doc, dtype=torch.int32))
        O.fill_(7.0)
        lse.fill_(7.0)
        graph.replay()
        assert B.samkv_poll_status(h) == 0
        check_prompt(q, k, v, new, dtype, mods, O, lse)


def test_two_handles_at_once():
    """Two streams, a handle each, the same inputs: every result as that of a call alone."""
    calls = []
    for dtype, kind in (("bf16", "cap+doc"), ("f32", "slope+window"), ("bf16", "window+prefix")):
        lens = [300, 1, 77, 500]
        q, k, v = (randn(sum(lens), h, 64, dtype=dtype, seed=i + 220) for i, h in enumerate((8, 2, 2)))
        mods = mods_of(kind, lens, [0] * 4, 8)
        want, _ = prompt(q, k, v, lens, dtype, mods)
        p = B.Packed(8, 2, 64, offsets_of(lens), sum(lens), 0, dtype)
        calls.append((B.Handle.for_scores(p), p, q, k, v, mods.device(B, DEV), torch.zeros_like(q), want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for h, p, q, k, v, scores, O, want, stream in calls:
            with torch.cuda.stream(stream):
                B.samkv_prefill_scores(h, p, q, k, v, 0.0, scores, O)
    torch.cuda.synchronize()
    for h, _, _, _, _, _, O, want, _ in calls:
        assert torch.equal(O, want) and B.samkv_poll_status(h) == 0


def test_workspaces():
    """A workspace of the plain calls is refused, one for the modified calls serves both."""
    lens = [500, 400]
    q, k, v = (randn(900, h, 64, seed=i + 230) for i, h in enumerate((8, 2, 2)))
    p = B.Packed(8, 2, 64, offsets_of(lens), 900)
    O, plain = torch.zeros_like(q), torch.zeros_like(q)
    with pytest.raises(B.SamkvError) as e:
        B.samkv_prefill_scores(B.Handle.for_packed(p), p, q, k, v, 0.0, B.Scores(softcap=5.0), O)
    assert e.value.status == 3
    assert B.samkv_scores_workspace_bytes(p) > B.samkv_packed_workspace_bytes(p)
    B.samkv_prefill(B.Handle.for_packed(p), p, q, k, v, 0.0, plain)
    h = B.Handle.for_scores(p)
    for _ in range(2):
        B.samkv_prefill_scores(h, p, q, k, v, 0.0, B.Scores(window=10), O)
        B.samkv_prefill(h, p, q, k, v, 0.0, O)
        assert torch.equal(O, plain)


def test_pages_without_cache_lengths_and_optional_outputs():
    p = B.Packed(2, 1, 64, torch.tensor([0, 3, 3, 40], dtype=torch.int32, device=DEV), 41)
    h = B.Handle.for_packed(p)
    table = torch.full((3, 4), -5, dtype=torch.int32, device=DEV)
    free, n = torch.tensor([7, 3, 5, 0, 1], dtype=torch.int32, device=DEV), torch.tensor([5], dtype=torch.int32, device=DEV)
    B.samkv_page_tables(h, p, None, 16, table, free, n, n)
    # (a pool of five pages has no page 5 and no page 7: the one is refused, the other not needed)
    assert table.tolist() == [[1, -5, -5, -5], [-5] * 4, [0, -1, 3, -5]] and int(n) == 1
    assert B.samkv_poll_status(h) == 7
    slots = torch.zeros(41, dtype=torch.int32, device=DEV)
    n.fill_(5)
    B.samkv_page_tables(h, p, None, 16, table, free, n, n, slots=slots)
    assert slots.tolist() == [16, 17, 18] + list(range(16)) + [-1] * 16 + list(range(48, 53)) + [-1]
    assert B.samkv_poll_status(h) == 7


def test_other_integer_types_and_tensors_are_refused_or_understood():
    p = B.Packed(2, 1, 64, torch.tensor([0, 1], dtype=torch.int32, device=DEV), 1)
    h = B.Handle.for_packed(p)
    table = torch.zeros((1, 2), dtype=torch.int32, device=DEV)
    free, n = torch.tensor([0, 1], dtype=torch.int32, device=DEV), torch.tensor([2], dtype=torch.int32, device=DEV)
    B.samkv_page_tables(h, p, None, np.int64(16), table, free, n, n)
    assert table.tolist() == [[1, 0]] and B.samkv_poll_status(h) == 0
    for bad in (free.long(), free.cpu(), torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)[::2]):
        with pytest.raises(ValueError):
            B.samkv_page_tables(h, p, None, 16, table, free, n, bad)
        with pytest.raises(ValueError):
            B.samkv_page_tables(h, p, bad, 16, table, free, n, n)
    with pytest.raises(ValueError):
        B.samkv_release_pages(h, table, 16, n, n, free, n, n)
    x = randn(1, 2, 64, seed=240)
    with pytest.raises(ValueError):
        B.samkv_prefill_scores(h, p, x, x[:, :1], x[:, :1], 0.0, B.Scores(slopes=torch.zeros(3, device=DEV)), torch.zeros_like(x))
    with pytest.raises(ValueError):
        B.samkv_prefill_scores(h, p, x.float(), x[:, :1], x[:, :1], 0.0, None, torch.zeros_like(x))


@pytest.mark.parametrize("dtype,n", [("bf16", 10500), ("f32", 5300)])
def test_plans_of_many_row_tiles(dtype, n):
    """Hundreds of row tiles with documents: the plan kernel goes through their tokens with several lanes each."""
    Hq, Hkv, d = 8, 2, 64
    q, k, v = (randn(n + 7, h, d, dtype=dtype, seed=i + 250) for i, h in enumerate((Hq, Hkv, Hkv)))
    r = np.random.default_rng(5)
    lens = [3, n - 3]
    p = np.concatenate([np.arange(x) for x in lens])
    doc = p // 777 * 777
    doc[n - 900:] = r.integers(-5, n, 900)                    # some tokens see nothing of their own
    mods = Mods(softcap=8.0, prefix=[1, 20], doc=np.concatenate([doc, np.zeros(7, dtype=np.int64)]))
    O, lse = prompt(q, k, v, lens, dtype, mods)
    rows = np.unique(np.concatenate([[0, 1, 776, 777, 778, 5000, n - 4, n - 904], r.integers(0, n - 3, 24), n - 4 - r.integers(0, 900, 16)]))
    ok = mods.seen(1, 3, 0, n - 3, n - 3)[rows]
    ref = attend64(f64(q)[3 + rows], f64(k)[3:n].swapaxes(0, 1), f64(v)[3:n].swapaxes(0, 1), ok, rows, mods, d ** -0.5)
    check(f64(O)[3 + rows], f64(lse)[3 + rows], ref, dtype, n)
    assert bool((O[n:] == 7.0).all())
