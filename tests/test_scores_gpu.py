"""samkv_prefill_scores and samkv_paged_attn_scores against the plain 64-bit form (scores_testlib)."""
import math

import numpy as np
import pytest
import torch

from paper_2508_11661_b200 import binding as B
from packed_testlib import DT, PagedCase, f64
from scores_testlib import Mods, attend64, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def offsets_of(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV)


def randn(*shape, dtype="bf16", seed=0, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * gain).to(DT[dtype]).to(DEV)


def slopes_of(n):
    return 2.0 ** (-8.0 * (np.arange(n) + 1) / n)


def mods_of(kind, lens, base, Hq, seed=0):
    """The modifications `kind` names, for sequences of these new tokens behind these slots."""
    r = np.random.default_rng(seed)
    kw = {}
    if "cap" in kind:
        kw["softcap"] = 5.0
    if "slope" in kind:
        kw["slopes"] = slopes_of(Hq)
    if "rising" in kind:
        kw["slopes"] = -slopes_of(Hq) * 0.1
    if "window" in kind:
        kw["window"] = 37
    if "prefix" in kind:
        kw["prefix"] = r.integers(0, 150, len(lens))
    if "doc" in kind:
        doc = []
        for n, c in zip(lens, base):
            borders = np.sort(r.integers(0, c + n + 1, 4))
            p = c + np.arange(n)
            d = np.array([max([0] + [b for b in borders if b <= x]) for x in p], dtype=np.int64)
            d[n - n // 8:] = 0                            # a question that sees all documents
            doc.append(d)
        kw["doc"] = np.concatenate(doc + [np.zeros(64, dtype=np.int64)])
    if "empty" in kind:                                   # some tokens see nothing
        doc = [np.where(r.random(n) < 0.5, 1 << 29, -5) for n in lens]
        kw["doc"] = np.concatenate(doc + [np.zeros(64, dtype=np.int64)])
    return Mods(**kw)


def prompt(q, k, v, lens, dtype, mods, scale=0.0, max_seq=0, handle=None, fill=7.0, want_lse=True):
    T, Hq, d = q.shape
    if mods.doc is not None:
        mods.doc = mods.doc[:T] if len(mods.doc) >= T else np.concatenate([mods.doc, np.zeros(T - len(mods.doc), dtype=np.int64)])
    p = B.Packed(Hq, k.shape[1], d, offsets_of(lens), T, max_seq, dtype)
    h = handle or B.Handle.for_scores(p)
    O = torch.full((T, Hq, d), fill, dtype=q.dtype, device=DEV)
    lse = torch.full((T, Hq), fill, dtype=torch.float32, device=DEV) if want_lse else None
    B.samkv_prefill_scores(h, p, q, k, v, scale, mods.device(B, DEV), O, lse)
    assert B.samkv_poll_status(h) == 0
    return O, lse


def check_prompt(q, k, v, lens, dtype, mods, O, lse, scale=0.0, fill=7.0):
    scale = scale if scale > 0 else 1.0 / math.sqrt(q.shape[2])
    q6, k6, v6, o6, l6 = f64(q), f64(k), f64(v), f64(O), f64(lse)
    at = 0
    for s, n in enumerate(lens):
        r = slice(at, at + n)
        ref = attend64(q6[r], k6[r].swapaxes(0, 1), v6[r].swapaxes(0, 1), mods.seen(s, at, 0, n, n), np.arange(n), mods, scale)
        check(o6[r], l6[r], ref, dtype, n, f"sequence {s} of {n}")
        at += n
    assert (o6[at:] == fill).all() and (l6[at:] == fill).all(), "rows behind the last sequence"


KINDS = ["cap", "slope", "rising", "window", "prefix", "doc", "empty", "cap+slope", "window+prefix", "doc+prefix+cap",
         "empty+prefix", "cap+slope+window+prefix+doc"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 64), (8, 2, 128)])
def test_prompts(dtype, kind, Hq, Hkv, d):
    lens = [1, 0, 2, 17, 128, 129, 0, 127, 300, 1, 64, 65, 31, 33, 32]
    T = sum(lens) + 5
    q, k, v = (randn(T, h, d, dtype=dtype, seed=i, gain=g) for i, (h, g) in enumerate(((Hq, 4.0), (Hkv, 1.0), (Hkv, 1.0))))
    mods = mods_of(kind, lens, [0] * len(lens), Hq)
    O, lse = prompt(q, k, v, lens, dtype, mods)
    check_prompt(q, k, v, lens, dtype, mods, O, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(3, 3, 128), (5, 1, 64), (32, 1, 128), (6, 2, 128), (16, 1, 64)])
@pytest.mark.parametrize("kind", ["cap+doc+prefix", "slope+window"])
def test_prompt_heads_and_lengths(dtype, Hq, Hkv, d, kind):
    for lens in ([700], [1], [1] * 40, [0, 9, 513, 255, 257]):
        T = sum(lens)
        q, k, v = (randn(T, h, d, dtype=dtype, seed=i + 5) for i, h in enumerate((Hq, Hkv, Hkv)))
        for max_seq in (0, max(lens), 1):                 # the hint chooses a kernel, never the result
            mods = mods_of(kind, lens, [0] * len(lens), Hq, seed=1)
            O, lse = prompt(q, k, v, lens, dtype, mods, max_seq=max_seq)
            check_prompt(q, k, v, lens, dtype, mods, O, lse)


def paged(c, mods, causal=True, scale=0.0, max_seq=0, handle=None, want_lse=True):
    p = B.Packed(c.Hq, c.Hkv, c.d, c.offsets, c.T, max_seq, c.dtype)
    h = handle or B.Handle.for_scores(p)
    if mods.doc is not None:
        mods.doc = np.concatenate([mods.doc, np.zeros(max(0, c.T - len(mods.doc)), dtype=np.int64)])[:c.T]
    O = torch.full((c.T, c.Hq, c.d), 7.0, dtype=DT[c.dtype], device=DEV)
    lse = torch.full((c.T, c.Hq), 7.0, dtype=torch.float32, device=DEV) if want_lse else None
    B.samkv_paged_attn_scores(h, p, B.Pages(c.Kp, c.Vp, c.table), c.cache_len, c.Q, scale, causal, mods.device(B, DEV), O, lse)
    assert B.samkv_poll_status(h) == 0
    return O, lse


def check_paged(c, mods, O, lse, causal=True, scale=0.0, sample=None):
    scale = scale if scale > 0 else 1.0 / math.sqrt(c.d)
    q6, o6, l6 = f64(c.Q), f64(O), f64(lse)
    for s, n in enumerate(c.new):
        L = c.cached[s] + n if causal else c.cached[s]
        at = int(c.starts[s])
        t = np.arange(n) if sample is None else np.unique(np.clip(sample, 0, n - 1)) if n else np.arange(0)
        ok = mods.seen(s, at, c.cached[s], n, L, causal)[t]
        ref = attend64(q6[at + t], c.slots(c.Kp, s, L), c.slots(c.Vp, s, L), ok, c.cached[s] + t, mods, scale)
        check(o6[at + t], l6[at + t], ref, c.dtype, max(L, 1), f"sequence {s}: {n} over {c.cached[s]}")
    assert (o6[c.total:] == 7.0).all() and (l6[c.total:] == 7.0).all(), "rows behind the last sequence"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("causal", [True, False])
def test_paged(dtype, kind, causal):
    new, cached = [1, 5, 0, 64, 1, 33, 1, 1, 20, 1], [700, 0, 9, 131, 15, 512, 0, 16, 63, 300]
    c = PagedCase(new, cached, 8, 2, 128, 16, dtype, seed=30, pad=3)
    c.Q *= 4
    mods = mods_of(kind, new, cached, 8, seed=2)
    O, lse = paged(c, mods, causal)
    check_paged(c, mods, O, lse, causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (8, 1, 64), (3, 3, 128), (5, 1, 64), (32, 2, 128)])
def test_decode(dtype, page, Hq, Hkv, d):
    cached = [0, 1, 15, 16, 63, 64, 65, 127, 128, 129, 1000, 255, 700]
    c = PagedCase([1] * len(cached), cached, Hq, Hkv, d, page, dtype, seed=31, garbage=float("nan"))
    for kind in ("cap", "slope", "window+prefix", "cap+slope+window+prefix+doc", "empty"):
        mods = mods_of(kind, c.new, cached, Hq, seed=3)
        for max_seq in (1, 0, 64):
            O, lse = paged(c, mods, max_seq=max_seq)
            check_paged(c, mods, O, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["cap", "slope", "window+prefix", "doc"])
def test_long_caches(dtype, kind):
    """One token over 30000 slots and a chunk over 9000 (work that is split along the cache), next to short ones."""
    new, cached = [1, 1, 150, 2], [30000, 5, 9000, 700]
    c = PagedCase(new, cached, 8, 2, 64, 64, dtype, seed=32)
    c.Q *= 4
    mods = mods_of(kind, new, cached, 8, seed=4)
    if mods.window:
        mods.window = 5000
    O, lse = paged(c, mods)
    check_paged(c, mods, O, lse, sample=[0, 1, 30, 63, 64, 127, 128, 149])
    again, lse2 = paged(c, mods)
    assert torch.equal(O, again) and torch.equal(lse, lse2), "results repeat bit for bit"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_prompt_of_documents(dtype):
    """Documents behind an instruction, a question behind them, in one sequence of many tiles; rows at the borders."""
    n, doc_len, pre, tail = 2900, 700, 40, 60
    Hq, Hkv, d = 8, 2, 64
    q, k, v = (randn(n, h, d, dtype=dtype, seed=i + 40, gain=g) for i, (h, g) in enumerate(((Hq, 4.0), (Hkv, 1.0), (Hkv, 1.0))))
    p = np.arange(n)
    doc = np.where(p >= pre, (p - pre) // doc_len * doc_len + pre, 0)
    doc[n - tail:] = 0
    mods = Mods(softcap=20.0, prefix=[pre], doc=doc)
    O, lse = prompt(q, k, v, [n], dtype, mods)
    rows = np.array(sorted({0, 1, 39, 40, 41, 127, 128, 739, 740, 741, 1439, 1440, 2000, 2139, 2140, 2839, 2840, 2899}))
    ref = attend64(f64(q)[rows], f64(k).swapaxes(0, 1), f64(v).swapaxes(0, 1), mods.seen(0, 0, 0, n, n)[rows], rows, mods, d ** -0.5)
    check(f64(O)[rows], f64(lse)[rows], ref, dtype, n)
    # the documents by themselves, as sequences of their own with the instruction in front of each: the same attention
    t = pre + doc_len + np.arange(10)
    own = np.concatenate([np.arange(pre), pre + doc_len + np.arange(10)])
    ref = attend64(f64(q)[t], f64(k)[own].swapaxes(0, 1), f64(v)[own].swapaxes(0, 1),
                   np.arange(len(own))[None, :] <= pre + np.arange(10)[:, None], pre + np.arange(10), mods, d ** -0.5)
    check(f64(O)[t], f64(lse)[t], ref, dtype, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["K", "V", "both"])
def test_hidden_slots_do_not_reach_a_row(dtype, bad, where):
    """Infinities and NaN before a document's start, outside a window, behind a prefix and behind the row itself."""
    lens, Hq, Hkv, d = [400, 300], 4, 2, 128
    T = sum(lens)
    q, k, v = (randn(T, h, d, dtype=dtype, seed=i + 50) for i, h in enumerate((Hq, Hkv, Hkv)))
    doc = np.concatenate([np.where(np.arange(400) >= 150, 150, 0), np.zeros(300, dtype=np.int64)])
    mods = Mods(window=100, prefix=[30, 0], doc=doc, softcap=10.0)
    O, lse = prompt(q, k, v, lens, dtype, mods)
    k2, v2 = k.clone(), v.clone()
    for x in ((k2,) if where == "K" else (v2,) if where == "V" else (k2, v2)):
        x[60:150, :, 3] = bad                             # seen by tokens 60 .. 149 of the first sequence
        x[400 + 120, :, 7] = bad                          # seen by tokens 120 .. 219 of the second
    O2, lse2 = prompt(q, k2, v2, lens, dtype, mods)
    keep = np.r_[0:60, 150:400, 400:520, 620:700]
    assert torch.equal(O[keep], O2[keep]) and torch.equal(lse[keep], lse2[keep])
    check_prompt(q, k2, v2, lens, dtype, mods, O2, lse2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_behind_a_window_may_be_gone(dtype):
    """Table entries of pages that no token sees hold anything; the pages they named hold NaN."""
    new, cached = [1, 1, 40, 1], [3000, 129, 700, 64]
    for page in (16, 64, 256):
        c = PagedCase(new, cached, 8, 2, 128, page, dtype, seed=60, garbage=float("nan"))
        mods = Mods(window=100, prefix=[20, 0, 5, 300], slopes=slopes_of(8))
        O, lse = paged(c, mods)
        check_paged(c, mods, O, lse)
        table = c.table.clone()
        for s in range(4):
            for col in range(c.width):
                lo, hi = col * page, (col + 1) * page
                first = max(0, cached[s] - 99)
                if not (hi > first and lo < cached[s] + new[s]) and not lo < mods.prefix[s]:
                    if lo < cached[s] + new[s]:
                        c.Kp[int(table[s, col])] = float("nan")
                        c.Vp[int(table[s, col])] = float("nan")
                    c.table[s, col] = [-1, 1 << 30, 0][col % 3]
        O2, lse2 = paged(c, mods)
        assert torch.equal(O, O2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_scores_are_capped(dtype):
    """A capped infinite score is the cap itself; without a cap it leaves NaN, as in the plain form."""
    n = 200
    q, k, v = (randn(n, 2, 64, dtype=dtype, seed=i + 70) for i in range(3))
    q[:, :, 0] = q[:, :, 0].abs() + 1.0
    k[20, 0, 0], k[40, 1, 0] = float("inf"), -float("inf")
    mods = Mods(softcap=4.0)
    O, lse = prompt(q, k, v, [n], dtype, mods)
    ok = mods.seen(0, 0, 0, n, n)
    # 2000 for the infinity: a score of 250 and more, whose tanh(x / 4) is 1 in 64 bits
    k6 = np.nan_to_num(f64(k), posinf=2000.0, neginf=-2000.0)
    ref = attend64(f64(q), k6.swapaxes(0, 1), f64(v).swapaxes(0, 1), ok, np.arange(n), mods, 64 ** -0.5)
    check(f64(O), f64(lse), ref, dtype, n)
    k[20, 0, 0] = float("nan")
    O, lse = prompt(q, k, v, [n], dtype, mods)
    assert bool(O[20:, 0].isnan().all()) and bool(O[:20].isfinite().all()) and bool(O[:, 1].isfinite().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [1e-3, 1.0, 1e6])
def test_extreme_caps_and_scales(dtype, cap):
    n = 260
    q, k, v = (randn(n, 4, 128, dtype=dtype, seed=i + 80, gain=8.0 if i == 0 else 1.0) for i in range(3))
    for scale in (0.0, 1.0):
        mods = Mods(softcap=cap, slopes=[0.0, 1.0, 1e-4, -0.01])
        O, lse = prompt(q, k, v, [n], dtype, mods, scale=scale)
        check_prompt(q, k, v, [n], dtype, mods, O, lse, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_modified_is_the_plain_call(dtype):
    lens = [40, 200, 7]
    T, Hq, Hkv, d = sum(lens), 8, 2, 128
    q, k, v = (randn(T, h, d, dtype=dtype, seed=i + 90) for i, h in enumerate((Hq, Hkv, Hkv)))
    p = B.Packed(Hq, Hkv, d, offsets_of(lens), T, 0, dtype)
    h = B.Handle.for_scores(p)
    O, O2 = torch.zeros_like(q), torch.zeros_like(q)
    B.samkv_prefill(h, p, q, k, v, 0.0, O)
    for scores in (None, B.Scores()):
        B.samkv_prefill_scores(h, p, q, k, v, 0.0, scores, O2)
        assert torch.equal(O, O2)
    # masks that hide nothing
    mods = Mods(window=1 << 30, prefix=[0, -7, 0], doc=np.full(T, -3))
    O3, lse = prompt(q, k, v, lens, dtype, mods)
    check_prompt(q, k, v, lens, dtype, Mods(), O3, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_optional_outputs(dtype):
    lens = [40, 200, 7]
    T, Hq, Hkv, d = sum(lens) + 6, 8, 2, 128
    fused = randn(T, Hq + 2 * Hkv, d, dtype=dtype, seed=95)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    mods = mods_of("cap+slope+window+prefix+doc", lens, [0] * 3, Hq, seed=5)
    O, lse = prompt(q, k, v, lens, dtype, mods)
    check_prompt(q, k, v, lens, dtype, mods, O, lse)
    O2, none = prompt(q, k, v, lens, dtype, mods, want_lse=False)
    assert none is None and torch.equal(O, O2)
    slab_k, slab_v = k.permute(1, 0, 2).contiguous(), v.permute(1, 0, 2).contiguous()
    O3, _ = prompt(q, slab_k.permute(1, 0, 2), slab_v.permute(1, 0, 2), lens, dtype, mods)
    assert torch.equal(O, O3)
    p = B.Packed(Hq, Hkv, d, offsets_of(lens), T, 0, dtype)
    wide = torch.full((T, Hq + 3, d), 5.0, dtype=DT[dtype], device=DEV)
    B.samkv_prefill_scores(B.Handle.for_scores(p), p, q, k, v, 0.0, mods.device(B, DEV), wide[:, 1:1 + Hq])
    n = sum(lens)
    assert torch.equal(wide[:n, 1:1 + Hq], O[:n]) and bool((wide[:, 0] == 5.0).all()) and bool((wide[n:] == 5.0).all())


def test_replay_with_other_lengths_and_masks():
    """A captured step is replayed after lengths, masks and slopes have changed; another call shares the handle in between."""
    for dtype in ("bf16", "f32"):
        c = PagedCase([1, 30, 1, 5], [600, 100, 0, 40], 8, 2, 128, 16, dtype, seed=100, spare_cols=4)
        p = B.Packed(8, 2, 128, c.offsets, c.T, 0, dtype)
        h = B.Handle.for_scores(p)
        mods = Mods(softcap=5.0, window=200, slopes=slopes_of(8), prefix=[3, 0, 9, 0], doc=np.zeros(c.T, dtype=np.int64))
        scores = mods.device(B, DEV)
        O, lse = torch.zeros_like(c.Q), torch.zeros((c.T, 8), device=DEV)
        pages = B.Pages(c.Kp, c.Vp, c.table)

        def call():
            B.samkv_paged_attn_scores(h, p, pages, c.cache_len, c.Q, 0.0, True, scores, O, lse)
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            call()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for k, (new, cached) in enumerate([([1, 30, 1, 5], [600, 100, 0, 40]), ([0, 1, 1, 35], [17, 128, 0, 9]), ([37, 0, 0, 0], [500, 1, 1, 1])]):
            c.new, c.cached = new, cached
            c.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
            c.offsets.copy_(torch.from_numpy(c.starts))
            c.cache_len.copy_(torch.tensor(cached, dtype=torch.int32))
            c.total = sum(new)
            mods.prefix = np.array([k, 5 * k, 2, 1])
            mods.doc = np.random.default_rng(k).integers(0, 50, c.T)
            mods.slopes = (slopes_of(8) * (k + 1)).astype(np.float32)
            scores.prefix_len.copy_(torch.tensor(mods.prefix, dtype=torch.int32))
            scores.doc_start.copy_(torch.tensor(mods.doc, dtype=torch.int32))
            scores.slopes.copy_(torch.from_numpy(mods.slopes))
            # every page that a row of the table may need is there
            order = torch.randperm(c.n_pages)[:c.n_pages].to(torch.int32)
            c.table_cpu = order[torch.arange(4 * c.width) % c.n_pages].reshape(4, c.width)
            c.table.copy_(c.table_cpu)
            O.fill_(7.0)
            lse.fill_(7.0)
            graph.replay()
            B.samkv_paged_attn(h, p, pages, c.cache_len, c.Q, 0.0, True, torch.empty_like(c.Q))
            assert B.samkv_poll_status(h) == 0
            check_paged(c, mods, O, lse)


def test_offsets_out_of_bounds_are_recorded():
    lens = [40, 30, 20]
    T = 90
    for dtype in ("bf16", "f32"):
        q, k, v = (randn(T, h, 64, dtype=dtype, seed=i + 110) for i, h in enumerate((4, 2, 2)))
        mods = Mods(softcap=5.0, window=10)
        good, lse = prompt(q, k, v, lens, dtype, mods)
        for off in ([0, 40, 30, 90], [-5, 40, 70, 90], [0, 40, 70, 1000]):
            p = B.Packed(4, 2, 64, torch.tensor(off, dtype=torch.int32, device=DEV), T, 0, dtype)
            h = B.Handle.for_scores(p)
            O = torch.full_like(q, 7.0)
            B.samkv_prefill_scores(h, p, q, k, v, 0.0, mods.device(B, DEV), O)
            assert B.samkv_poll_status(h) == 7 and B.samkv_poll_status(h) == 0
            assert torch.equal(O[:40], good[:40])
            if off[2] == 30:                              # it ends the list
                assert bool((O[40:] == 7.0).all())
            B.samkv_prefill_scores(h, B.Packed(4, 2, 64, offsets_of(lens), T, 0, dtype), q, k, v, 0.0, mods.device(B, DEV), O)
            assert B.samkv_poll_status(h) == 0 and torch.equal(O, good)


def test_a_page_that_is_none_is_recorded():
    for new in ([1, 1], [40, 1]):
        c = PagedCase(new, [100, 50], 8, 2, 128, 16, "bf16", seed=120)
        c.table[0, 6] = 1 << 20
        p = B.Packed(8, 2, 128, c.offsets, c.T, max(new), "bf16")
        h = B.Handle.for_scores(p)
        O = torch.zeros_like(c.Q)
        B.samkv_paged_attn_scores(h, p, B.Pages(c.Kp, c.Vp, c.table), c.cache_len, c.Q, 0.0, True, B.Scores(softcap=5.0), O)
        assert B.samkv_poll_status(h) == 7 and B.samkv_poll_status(h) == 0


def test_many_sequences():
    """More sequences than a block has threads, most of them of one token."""
    r = np.random.default_rng(7)
    new = [int(x) for x in r.choice([0, 1, 1, 1, 3], 1500)]
    cached = [int(x) for x in r.integers(0, 60, 1500)]
    for dtype in ("bf16", "f32"):
        c = PagedCase(new, cached, 4, 2, 64, 16, dtype, seed=130, pad=2)
        mods = mods_of("cap+window+prefix+doc", new, cached, 4, seed=8)
        mods.prefix = r.integers(0, 30, 1500)
        for max_seq in (0, 3):
            O, lse = paged(c, mods, max_seq=max_seq)
            check_paged(c, mods, O, lse)


def test_other_streams():
    """The call runs on the current stream behind what was queued there."""
    c = PagedCase([1] * 8, [300] * 8, 8, 2, 128, 16, "bf16", seed=140)
    mods = Mods(softcap=5.0, window=64)
    p = B.Packed(8, 2, 128, c.offsets, c.T, 1, "bf16")
    h = B.Handle.for_scores(p)
    want, _ = paged(c, mods)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    scores, pages, O = mods.device(B, DEV), B.Pages(c.Kp, c.Vp, c.table), torch.zeros_like(c.Q)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for i in range(50):
            q = (c.Q * 0 if i % 2 else c.Q).clone()       # written right before the call
            B.samkv_paged_attn_scores(h, p, pages, c.cache_len, q, 0.0, True, scores, O)
            if i % 2 == 0:
                assert torch.equal(O, want)
    stream.synchronize()
