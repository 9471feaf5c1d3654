"""samkv_page_tables, samkv_release_pages and samkv_append_axes against plain forms, and the step they make together with
attention."""
import math

import numpy as np
import pytest
import torch

from paper_2508_11661_b200 import binding as B
from packed_testlib import DT, PagedCase, f64, rotate64, rotate_bound
from scores_testlib import Mods, attend64, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Host:
    """The page pool on the host: a stack and a table, changed one page at a time."""

    def __init__(self, n_seq, width, page, n_pages, seed=0):
        r = np.random.default_rng(seed)
        self.page, self.width, self.n_pages = page, width, n_pages
        self.stack = [int(x) for x in r.permutation(n_pages)]
        self.table = np.full((n_seq, width), -7, dtype=np.int64)
        self.lens = [0] * n_seq
        self.full = False

    def step(self, new, n_tokens):
        slots, positions, at = [-1] * n_tokens, [0] * n_tokens, 0
        total = list(self.lens)
        for s, n in enumerate(new):
            for t in range(n):
                pos = self.lens[s] + t
                if pos >= self.width * self.page:
                    self.full = True
                else:
                    if pos % self.page == 0:
                        self.table[s, pos // self.page] = self.stack.pop() if self.stack else -1
                    page = self.table[s, pos // self.page]
                    if page >= 0:
                        slots[at] = page * self.page + pos % self.page
                        total[s] = pos + 1
                    else:
                        self.full = True
                positions[at] = pos
                at += 1
        self.lens = total
        return slots, positions

    def release(self, done):
        for s in reversed(range(len(done))):
            if done[s]:
                self.stack += [int(x) for x in self.table[s, :-(-self.lens[s] // self.page)][::-1]]
                self.lens[s] = 0


class Device:
    def __init__(self, host):
        self.table = dev32(host.table)
        self.free = dev32(host.stack + [-9] * (host.n_pages - len(host.stack)))
        self.n_free = dev32([len(host.stack)])
        self.lens = dev32(host.lens)
        self.host = host

    def step(self, new, n_tokens, out=None, offsets=None, handle=None):
        h = self.host
        p = B.Packed(2, 1, 64, dev32(np.concatenate([[0], np.cumsum(new)])) if offsets is None else offsets, n_tokens)
        handle = handle or B.Handle.for_packed(p)
        slots, positions, total = (torch.full((n,), 55, dtype=torch.int32, device=DEV) for n in (n_tokens, n_tokens, len(new)))
        B.samkv_page_tables(handle, p, self.lens, h.page, self.table, self.free, self.n_free, self.n_free if out is None else out,
                            slots, positions, total)
        self.lens = total
        return slots.tolist(), positions.tolist(), B.samkv_poll_status(handle)

    def release(self, done, out=None):
        p = B.Packed(2, 1, 64, dev32([0, 0]), 0)
        handle = B.Handle.for_packed(p)
        done = torch.tensor(done, device=DEV)
        B.samkv_release_pages(handle, self.table, self.host.page, self.lens, done, self.free, self.n_free,
                              self.n_free if out is None else out)
        self.lens = torch.where(done.bool(), 0, self.lens).to(torch.int32)
        return B.samkv_poll_status(handle)

    def same(self):
        h = self.host
        assert self.lens.tolist() == h.lens
        n = int(self.n_free)
        assert n == len(h.stack) and self.free[:n].tolist() == h.stack
        assert np.array_equal(self.table.cpu().numpy(), h.table)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("n_seq", [1, 7, 300, 1700])
def test_steps_of_growing_and_finishing_requests(page, n_seq):
    r = np.random.default_rng(page + n_seq)
    h = Host(n_seq, 3000 // page + 4, page, 12 * n_seq * max(1, 64 // page) + 200, seed=n_seq)
    d = Device(h)
    for k in range(6):
        new = [int(x) for x in r.choice([0, 1, 1, 1, 5, page, 2 * page + 3], n_seq)]
        if k % 2:
            new = [1] * n_seq
        T = sum(new) + int(r.integers(0, 9))
        want = h.step(new, T)
        slots, positions, status = d.step(new, T)
        assert status == (7 if h.full else 0)
        assert slots == want[0] and positions == want[1]
        d.same()
        h.full = False
        done = [bool(x) for x in r.random(n_seq) < 0.2]
        h.release(done)
        assert d.release(done) == 0
        d.same()


@pytest.mark.parametrize("n_seq,long", [(1, 90000), (3, 20000), (40, 3000)])
def test_long_prompts(n_seq, long):
    h = Host(n_seq, long // 64 + 3, 64, n_seq * (long // 64 + 2), seed=1)
    d = Device(h)
    for new in ([long - 7 * s for s in range(n_seq)], [1] * n_seq, [0] * n_seq):
        want = h.step(new, sum(new) + 3)
        got = d.step(new, sum(new) + 3)
        assert got[0] == want[0] and got[1] == want[1] and got[2] == 0
        d.same()


def test_empty_steps():
    h = Host(5, 4, 16, 9)
    d = Device(h)
    h.step([3, 0, 20, 0, 0], 23)
    d.step([3, 0, 20, 0, 0], 23)
    for T in (0, 6):                                      # no tokens, and only rows of no sequence
        assert d.step([0] * 5, T)[:2] == ([-1] * T, [0] * T)
        d.same()
    assert d.release([False] * 5) == 0
    d.same()


def test_pages_run_out_and_come_back():
    h = Host(4, 10, 16, 6, seed=3)
    d = Device(h)
    new = [17, 60, 5, 100]                                # 2 + 4 pages, then none
    want = h.step(new, 190)
    slots, positions, status = d.step(new, 190)
    assert status == 7 and slots == want[0] and positions == want[1]
    d.same()
    assert h.lens == [17, 60, 0, 0]
    want = h.step([14, 4, 0, 0], 18)                      # room in the last pages
    assert d.step([14, 4, 0, 0], 18) == (want[0], want[1], 0)
    d.same()
    h.release([False, True, False, False])
    assert d.release([False, True, False, False]) == 0
    d.same()
    want = h.step([0, 0, 5, 30], 35)
    assert d.step([0, 0, 5, 30], 35) == (want[0], want[1], 0)
    d.same()


def test_the_table_ends():
    h = Host(2, 2, 16, 9, seed=4)
    d = Device(h)
    want = h.step([40, 3], 43)
    slots, positions, status = d.step([40, 3], 43)
    assert status == 7 and slots == want[0] and positions == want[1]
    d.same()
    assert h.lens == [32, 3]


def test_counts_beside_one_another():
    """n_free_out elsewhere: the count stays, and the same call gives the same answer again."""
    h = Host(300, 8, 16, 2000, seed=5)
    d, out = Device(h), dev32([0])
    h.step([20] * 300, 6000)
    before, lens = d.n_free.clone(), d.lens
    for _ in range(3):
        d.lens = lens
        d.step([20] * 300, 6000, out=out)
        assert torch.equal(d.n_free, before) and int(out) == len(h.stack)
        assert np.array_equal(d.table.cpu().numpy(), h.table)
    d.n_free.copy_(out)
    done = [s % 3 == 0 for s in range(300)]
    h.release(done)
    lens, kept = d.lens, int(out)
    for _ in range(3):
        d.lens = lens
        assert d.release(done, out=out) == 0
        assert int(out) == len(h.stack) and int(d.n_free) == kept
    assert d.free[:int(out)].tolist() == h.stack


def test_bad_lists_and_lengths_are_recorded():
    h = Host(3, 4, 16, 8, seed=6)
    d = Device(h)
    d.n_free.fill_(99)                                    # clamped to the stack
    assert d.step([1, 1, 1], 3)[2] == 7 and int(d.n_free) == 5
    d = Device(h)
    d.n_free.fill_(-4)
    slots, _, status = d.step([1, 1, 1], 3)
    assert status == 7 and slots == [-1] * 3 and int(d.n_free) == 0 and d.lens.tolist() == [0] * 3
    d = Device(h)
    d.free[7] = 8                                         # no page; the others get theirs
    slots, _, status = d.step([1, 1, 1], 3)
    assert status == 7 and slots == [-1] + [16 * h.stack[6], 16 * h.stack[5]] and d.table[0, 0] == -1
    d = Device(h)
    d.lens = dev32([5, 0, 0])                             # a length whose page is not in the table
    slots, _, status = d.step([1, 0, 0], 1)
    assert status == 7 and slots == [-1]
    d = Device(h)
    d.lens = dev32([1 << 20, -3, 0])
    assert d.release([True, True, False]) == 7            # clamped; more than the stack holds is dropped
    assert int(d.n_free) == 8 and d.free.tolist() == h.stack


@pytest.mark.parametrize("off", [[0, 4, 2, 6], [3, 1, 4, 6], [-2, 4, 5, 9], [2, 2, 5, 40]])
def test_offsets_out_of_order_or_bounds(off):
    """The rule of samkv_prefill: the list ends with a sequence that ends before it starts; the others are cut to the rows."""
    h = Host(3, 4, 16, 30, seed=7)
    d = Device(h)
    T, new, ended = 6, [], False
    for s in range(3):
        ended = ended or off[s + 1] < off[s]
        a = min(max(off[s], 0), T)
        new.append(0 if ended else min(max(off[s + 1], a), T) - a)
    first = min(max(off[0], 0), T)
    want = h.step(new, sum(new))
    pad = T - first - sum(new) if any(new) else T - first
    slots, positions, status = d.step([0] * 3, T, offsets=dev32(off))
    assert status == 7
    assert slots == [-1] * first + want[0] + [-1] * pad and positions == [0] * first + want[1] + [0] * pad
    d.same()


def test_captured_decode_steps():
    """Hand-out and release in one captured step, replayed while requests grow and finish."""
    n_seq, page = 40, 16
    h = Host(n_seq, 8, page, 300, seed=8)
    d = Device(h)
    h.step([10] * n_seq, 10 * n_seq)
    d.step([10] * n_seq, 10 * n_seq)
    p = B.Packed(2, 1, 64, dev32(range(n_seq + 1)), n_seq)
    handle = B.Handle.for_packed(p)
    slots, positions, total = (torch.zeros(n_seq, dtype=torch.int32, device=DEV) for _ in range(3))
    lens, done = d.lens.clone(), torch.zeros(n_seq, dtype=torch.bool, device=DEV)

    def step():
        B.samkv_release_pages(handle, d.table, page, lens, done, d.free, d.n_free, d.n_free)
        lens.masked_fill_(done, 0)
        B.samkv_page_tables(handle, p, lens, page, d.table, d.free, d.n_free, d.n_free, slots, positions, total)
        lens.copy_(total)
    state = [x.clone() for x in (d.table, d.free, d.n_free, lens)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, y in zip((d.table, d.free, d.n_free, lens), state):
        x.copy_(y)
    r = np.random.default_rng(9)
    for k in range(25):
        flags = r.random(n_seq) < 0.1
        done.copy_(torch.tensor(flags))
        h.release(list(flags))
        want = h.step([1] * n_seq, n_seq)
        graph.replay()
        assert slots.tolist() == want[0] and positions.tolist() == want[1]
        d.lens = lens
        d.same()
    assert B.samkv_poll_status(handle) == 0


# ------------------------------------------------------------------------------------------------ several axes
def slots_of(c, pad_to=None):
    out = []
    for s, n in enumerate(c.new):
        for t in range(n):
            j = c.cached[s] + t
            out.append(int(c.table_cpu[s, j // c.page]) * c.page + j % c.page)
    return out + [-1] * (c.T - len(out))


def rotate_axes(x, pos, axis, rot, base, interleaved, inv_freq=None):
    """pos [axes, n]: every axis's rotation by itself, of which each pair takes its own."""
    out = x.copy()
    half = rot // 2
    for a in range(pos.shape[0]):
        y = rotate64(x, pos[a], rot, base, interleaved, inv_freq)
        for i in range(half):
            if axis[i] == a:
                for e in ((2 * i, 2 * i + 1) if interleaved else (i, i + half)):
                    out[..., e] = y[..., e]
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 64), (6, 2, 128), (5, 1, 128)])
@pytest.mark.parametrize("rot,interleaved,axes", [(0, False, 1), (64, False, 3), (64, True, 2), (16, False, 4), (48, True, 3)])
@pytest.mark.parametrize("mapped", [True, False])
def test_append_axes(dtype, Hq, Hkv, d, rot, interleaved, axes, mapped):
    c = PagedCase([1, 0, 5, 130, 1, 17], [0, 9, 15, 33, 16, 1000], Hq, Hkv, d, 32, dtype, seed=20, pad=4)
    r = np.random.default_rng(rot)
    axis = [int(a) for a in r.integers(0, axes, rot // 2)]
    if rot:
        axis[:axes] = range(axes)
    pos = r.integers(-5000, 3_000_000, (axes, c.T))
    pos[:, :3] = [[2 ** 31 - 1, -2 ** 31, 0]]
    rope = B.RopeAxes(rot, axis, 500000.0, interleaved) if rot else None
    p = B.Packed(Hq, Hkv, d, c.offsets, c.T, 0, dtype)
    h = B.Handle.for_packed(p)
    K0, V0 = f64(c.Kp), f64(c.Vp)
    Q_out, K_out, V_out = torch.full_like(c.Q, 3.0), torch.full_like(c.K, 3.0), torch.full_like(c.V, 3.0)
    slots = slots_of(c)
    if mapped:
        slots[2] = -1                                     # left out altogether
        slots[7] = -(1 << 31)
    B.samkv_append_axes(h, p, c.K, c.V, B.Pages(c.Kp, c.Vp, c.table), None if mapped else c.cache_len,
                        dev32(slots) if mapped else None, rope, dev32(pos) if rot else None, c.Q, Q_out, K_out, V_out)
    assert B.samkv_poll_status(h) == 0
    k, v, q = f64(c.K), f64(c.V), f64(c.Q)
    if rot:
        kr, qr = (rotate_axes(x, pos, axis, rot, 500000.0, interleaved) for x in (k, q))
        kt, qt = rotate_bound(k, kr, rot, interleaved, dtype), rotate_bound(q, qr, rot, interleaved, dtype)
        kt[..., rot:], qt[..., rot:] = 0.0, 0.0
    else:
        kr, qr, kt, qt = k, q, 0 * k, 0 * q
    live = np.array([x >= 0 for x in slots])
    for got, want, tol in ((f64(Q_out), qr, qt), (f64(K_out), kr, kt), (f64(V_out), v, 0 * v)):
        assert (np.abs(got - want)[live] <= tol[live]).all() and (got[~live] == 3.0).all()
    tK = np.zeros_like(K0)
    for t in np.flatnonzero(live):
        page, row = slots[t] // c.page, slots[t] % c.page
        K0[page, :, row], V0[page, :, row], tK[page, :, row] = kr[t], v[t], kt[t]
    assert np.array_equal(f64(c.Vp), V0) and (np.abs(f64(c.Kp) - K0) <= tK).all()


def test_axes_that_agree_are_one_axis():
    """Text: the same bits as samkv_append, with positions given once, on every axis, or taken from the cache's lengths."""
    c = PagedCase([1, 40, 300], [100, 0, 7], 6, 2, 128, 16, "bf16", seed=21, pad=2)
    p = B.Packed(6, 2, 128, c.offsets, c.T, 0, "bf16")
    h = B.Handle.for_packed(p)
    pages = B.Pages(c.Kp, c.Vp, c.table)
    Q0 = torch.zeros_like(c.Q)
    B.samkv_append(h, p, c.K, c.V, pages, c.cache_len, B.Rope(128, 10000.0), None, c.Q, Q0)
    K0, V0 = c.Kp.clone(), c.Vp.clone()
    pos = dev32(np.concatenate([np.arange(a, a + n) for a, n in zip(c.cached, c.new)] + [np.zeros(2, dtype=np.int64)]))
    three = B.RopeAxes.sections([16, 24, 24], 10000.0)
    assert three.n_axes == 3 and list(three._axis)[15:17] == [0, 1]
    for rope in (three, B.RopeAxes(128, [0] * 64, 10000.0), B.RopeAxes(128, [i % 4 for i in range(64)], 10000.0)):
        for positions in (None, pos, pos[None].expand(4, -1).contiguous()):
            for slots in (None, dev32(slots_of(c))):
                if positions is None and slots is not None:
                    continue
                c.Kp.zero_(), c.Vp.zero_()
                c.Kp.copy_(K0), c.Vp.copy_(V0)
                for s, n in enumerate(c.new):             # what the call has to write is gone
                    for t in range(n):
                        j = c.cached[s] + t
                        c.Kp[int(c.table_cpu[s, j // 16]), :, j % 16] = 9.0
                Q = torch.zeros_like(c.Q)
                B.samkv_append_axes(h, p, c.K, c.V, pages, c.cache_len, slots, rope, positions, c.Q, Q)
                assert torch.equal(Q, Q0) and torch.equal(c.Kp, K0) and torch.equal(c.Vp, V0)
    assert B.samkv_poll_status(h) == 0


def test_a_slot_behind_the_pool_is_recorded():
    c = PagedCase([3], [0], 4, 2, 64, 16, "f32", seed=22)
    p = B.Packed(4, 2, 64, c.offsets, c.T, 0, "f32")
    h = B.Handle.for_packed(p)
    K0 = c.Kp.clone()
    for bad in (c.n_pages * 16, 2 ** 31 - 1):
        B.samkv_append_axes(h, p, c.K, c.V, B.Pages(c.Kp, c.Vp, c.table), slots=dev32([bad, -1, -1]))
        assert B.samkv_poll_status(h) == 7 and torch.equal(c.Kp, K0)


def test_rows_in_place():
    c = PagedCase([70], [3], 4, 2, 128, 64, "bf16", seed=23)
    p = B.Packed(4, 2, 128, c.offsets, c.T, 0, "bf16")
    h = B.Handle.for_packed(p)
    pos = dev32(np.random.default_rng(0).integers(0, 500, (2, 70)))
    rope, pages = B.RopeAxes(128, [i % 2 for i in range(64)]), B.Pages(c.Kp, c.Vp, c.table)
    Q, K_out, V_out = torch.zeros_like(c.Q), torch.zeros_like(c.K), torch.zeros_like(c.V)
    B.samkv_append_axes(h, p, c.K, c.V, pages, c.cache_len, None, rope, pos, c.Q, Q, K_out, V_out)
    q, k = c.Q.clone(), c.K.clone()
    B.samkv_append_axes(h, p, k, c.V, pages, None, dev32(slots_of(c)), rope, pos, q, q, k, c.V)
    assert torch.equal(q, Q) and torch.equal(k, K_out) and B.samkv_poll_status(h) == 0


# ------------------------------------------------------------------------------------------------ the step as a whole
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("captured", [False, True])
def test_serving_steps(dtype, captured):
    """Prompts with images, then decode steps, requests that finish and new ones in their place: pages from lengths, append by
    the slot map with three axes, attention with a cap, a window and initial tokens, all on the device; against a dense model."""
    Hq, Hkv, d, page, n_seq = 8, 2, 64, 16, 5
    r = np.random.default_rng(11)
    axis = [0] * 8 + [1] * 12 + [2] * 12
    rope = B.RopeAxes(d, axis, 10000.0)
    host = Host(n_seq, 20, page, 64, seed=12)
    host.table[:] = -1                                    # (a fresh device table says so too)
    dv = Device(host)
    Kp = torch.full((64, Hkv, page, d), float("nan"), dtype=DT[dtype], device=DEV)
    Vp = Kp.clone()
    T = 160
    offsets, positions = torch.zeros(n_seq + 1, dtype=torch.int32, device=DEV), torch.zeros((3, T), dtype=torch.int32, device=DEV)
    p = B.Packed(Hq, Hkv, d, offsets, T, 0, dtype)
    h = B.Handle.for_scores(p)
    pages = B.Pages(Kp, Vp, dv.table)
    scores = B.Scores(softcap=10.0, window=60, prefix_len=dev32([4] * n_seq))
    mods = Mods(softcap=10.0, window=60, prefix=[4] * n_seq)
    slots, pos_out, total = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (T, T, n_seq))
    lens, done = torch.zeros(n_seq, dtype=torch.int32, device=DEV), torch.zeros(n_seq, dtype=torch.bool, device=DEV)
    Q, K, V = (torch.zeros((T, x, d), dtype=DT[dtype], device=DEV) for x in (Hq, Hkv, Hkv))
    Qr, O, lse = torch.zeros_like(Q), torch.zeros_like(Q), torch.zeros((T, Hq), device=DEV)

    def step():
        B.samkv_release_pages(h, dv.table, page, lens, done, dv.free, dv.n_free, dv.n_free)
        lens.masked_fill_(done, 0)
        B.samkv_page_tables(h, p, lens, page, dv.table, dv.free, dv.n_free, dv.n_free, slots, pos_out, total)
        B.samkv_append_axes(h, p, K, V, pages, None, slots, rope, positions, Q, Qr)
        B.samkv_paged_attn_scores(h, p, pages, lens, Qr, 0.0, True, scores, O, lse)
        lens.copy_(total)
    graph = None
    if captured:
        state = [x.clone() for x in (dv.free, dv.n_free)]
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step()                                        # (no tokens yet: nothing changes)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for x, y in zip((dv.free, dv.n_free), state):
            x.copy_(y)
    keys = [np.zeros((0, Hkv, d)) for _ in range(n_seq)]
    values = [np.zeros((0, Hkv, d)) for _ in range(n_seq)]
    for k in range(8):
        new = [40, 17, 1, 0, 90] if k == 0 else [1, 1, 1, 33 if k == 3 else 0, 1]
        flags = [k == 5 and s == 4 for s in range(n_seq)]
        if k == 5:
            new[4] = 70                                   # another request takes the row
        host.release(flags)
        want = host.step(new, T)
        offsets.copy_(dev32(np.concatenate([[0], np.cumsum(new)])))
        done.copy_(torch.tensor(flags))
        pos = r.integers(0, 200, (3, T))
        positions.copy_(dev32(pos))
        for x, gain in ((Q, 3.0), (K, 1.0), (V, 1.0)):
            x.copy_(torch.from_numpy(r.normal(size=x.shape) * gain).to(DT[dtype]))
        O.fill_(7.0)
        step() if graph is None else graph.replay()
        assert B.samkv_poll_status(h) == 0
        assert slots.tolist() == want[0] and total.tolist() == host.lens
        # the dense model rounds the rotated rows as the cache does; what that rounding may differ by is the rotation's own test
        q6, v6 = f64(Qr), f64(V)
        k_rot = rotate_axes(f64(K), pos, axis, d, 10000.0, False)
        cache = f64(Kp)
        at = 0
        for s, n in enumerate(new):
            if flags[s]:
                keys[s], values[s] = keys[s][:0], values[s][:0]
            rows = np.arange(at, at + n)
            stored = np.array([cache[x // page, :, x % page] for x in np.array(want[0])[rows]]).reshape(n, Hkv, d)
            assert (np.abs(stored - k_rot[rows]) <= rotate_bound(f64(K)[rows], k_rot[rows], d, False, dtype)).all()
            base = len(keys[s])
            keys[s], values[s] = np.concatenate([keys[s], stored]), np.concatenate([values[s], v6[rows]])
            ok = mods.seen(s, at, base, n, base + n)
            ref = attend64(q6[rows], keys[s].swapaxes(0, 1), values[s].swapaxes(0, 1), ok, base + np.arange(n), mods, d ** -0.5)
            check(f64(O)[rows], f64(lse)[rows], ref, dtype, max(1, base + n), f"step {k}, sequence {s}")
            at += n
        assert bool((O[at:] == 7.0).all())
