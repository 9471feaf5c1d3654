"""Packed and paged calls where their rounding, their bounds and their hand-overs are easiest to get wrong."""
import numpy as np
import pytest
import torch

from paper_2508_11661_b200 import binding as B
from packed_testlib import DT, PagedCase, attend64, check_rows, f64
from test_packed_gpu import DEV, run_paged

pytestmark = pytest.mark.gpu


class FullTables(PagedCase):
    """Every sequence owns `width` pages, all of them filled; lengths are set by the test."""

    def __init__(self, new, width, Hq, Hkv, d, page, dtype, seed=0, pad=0):
        super().__init__(new, [0] * len(new), Hq, Hkv, d, page, dtype, seed=seed, pad=pad)
        g = torch.Generator().manual_seed(seed + 1000)
        self.width, self.n_pages = width, len(new) * width
        self.table_cpu = torch.randperm(self.n_pages, generator=g).to(torch.int32).view(len(new), width).contiguous()
        self.table = self.table_cpu.to(DEV)
        self.Kp = torch.randn((self.n_pages, Hkv, page, d), generator=g).to(DT[dtype]).to(DEV)
        self.Vp = torch.randn((self.n_pages, Hkv, page, d), generator=g).to(DT[dtype]).to(DEV)


# ------------------------------------------------------------------------------------------------ tables that are too short
@pytest.mark.parametrize("dtype,new,width,page,hint", [
    ("bf16", [3, 2, 3, 1, 3], 4, 16, 3),                 # decode
    ("bf16", [40, 7, 130, 300, 33], 3, 64, 0),           # tensor memory; 300 tokens pass a table of 192 slots by themselves
    ("f32", [3, 2, 3, 1, 3], 4, 16, 3),                  # 8 rows
    ("f32", [40, 7, 230, 300, 333], 3, 64, 0)])          # 64 rows
@pytest.mark.parametrize("causal", [True, False])
def test_sequences_that_pass_their_table_are_cut_off(dtype, new, width, page, hint, causal):
    """Token t sees the slots < cache_len + t + 1 (or < cache_len) as far as the table goes: a token that fits keeps its own."""
    limit = width * page
    for lens in ([limit - 1, limit, limit - 2, limit + 7, 0], [2**31 - 1, limit - 5, 1, 0, limit - 1]):
        c = FullTables(new, width, 8, 2, 128, page, dtype, seed=200, pad=3)
        c.cache_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
        over = any(n > limit or (causal and n + k > limit) for n, k in zip(lens, new))
        assert over
        O, lse = run_paged(c, causal, max_seq=hint, poll=7)
        q, o, l = f64(c.Q), f64(O), f64(lse)
        at = 0
        for s, n in enumerate(new):
            vis = np.minimum(lens[s] + (np.arange(1, n + 1) if causal else np.zeros(n, dtype=np.int64)), limit)
            ref = attend64(q[at:at + n], c.slots(c.Kp, s, limit), c.slots(c.Vp, s, limit), vis, 128 ** -0.5)
            check_rows(o[at:at + n], l[at:at + n], ref, dtype, limit, f"sequence {s}: {n} over {lens[s]} of {limit}")
            at += n
        assert (o[at:] == 7.0).all()


# ------------------------------------------------------------------------------------------------ offsets that run backwards
@pytest.mark.parametrize("dtype,hint,span", [("bf16", 2, 2), ("bf16", 0, 20), ("f32", 2, 2), ("f32", 0, 20)])
@pytest.mark.parametrize("n_seq,at", [(5, 1), (32, 31), (33, 7), (300, 150), (513, 2), (1200, 1000)])
def test_a_sequence_that_ends_before_it_starts_ends_the_list(dtype, hint, span, n_seq, at):
    """Those behind it start over on rows that others own: they are empty, the ones before it are what they are alone."""
    new = [span] * n_seq
    c = PagedCase(new, [30] * n_seq, 4, 2, 64, 16, dtype, seed=240)
    off = np.arange(n_seq + 1) * span
    off[at + 1:] -= min(off[at], span) + 1               # sequence `at` runs backwards, the next ones own rows twice
    assert (np.diff(off) < 0).sum() == 1 and off.min() >= 0
    good, good_lse = run_paged(c, max_seq=hint)
    c.offsets = torch.from_numpy(off.astype(np.int32)).to(DEV)
    O, lse = run_paged(c, max_seq=hint, poll=7)
    rows = at * span
    assert bool((O[rows:] == 7.0).all()) and bool((lse[rows:] == 7.0).all())
    # another division of the keys may round otherwise, by no more than the two results' own bounds
    tol = 2.0 ** -6 if dtype == "bf16" else 1e-5
    assert bool(((O[:rows] - good[:rows]).float().abs() <= tol * good.abs().amax().float()).all())
    assert bool((lse[:rows] - good_lse[:rows]).abs().le(1e-5).all())


# ------------------------------------------------------------------------------------------------ handles
def test_a_handle_made_behind_pending_work_of_its_workspace():
    """The allocator hands out memory that queued work of the same stream still writes; the handle's status block has to be
    cleared behind that work."""
    c = PagedCase([1], [9001], 8, 1, 128, 64, "bf16", seed=66)
    ref, _ = run_paged(c)
    p = B.Packed(c.Hq, c.Hkv, c.d, c.offsets, c.T, 0, c.dtype)
    nbytes = B.samkv_packed_workspace_bytes(p)
    pages = B.Pages(c.Kp, c.Vp, c.table)
    O = torch.full_like(c.Q, 7.0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        junk = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
        where = junk.data_ptr()
        for _ in range(1500):
            junk.fill_(255)
        del junk
        h = B.Handle.for_packed(p)
        assert h.workspace.data_ptr() == where
        B.samkv_paged_attn(h, p, pages, c.cache_len, c.Q, 0.0, True, O)
        assert B.samkv_poll_status(h) == 0
    assert torch.equal(O, ref)
