"""Packed and paged calls where their rounding, their bounds and their hand-overs are easiest to get wrong."""
import math

import numpy as np
import pytest
import torch

from paper_2508_11661_b200 import binding as B
from packed_testlib import DT, HALF_STEP, PagedCase, attend64, check_rows, f64, rotate_bound
from test_packed_gpu import DEV, check_paged, check_prefill, randn, run_paged, run_prefill

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


# ------------------------------------------------------------------------------------------------ rounding
def tight_bound(q, k, v, vis, scale, O, Es, A, length):
    """With a denominator that sums the very probabilities the product uses, their rounding errors e_j (half a step of 8
    bits) move the result by sum_j w_j e_j (v_j - O) / (1 + sum_j w_j e_j): values that agree are not moved at all."""
    n, Hq, d = q.shape
    G = Hq // k.shape[0]
    spread = np.zeros_like(O)
    for t in range(n):
        L = int(vis[t])
        for h in range(k.shape[0]):
            rows = slice(h * G, (h + 1) * G)
            x = q[t, rows] @ k[h, :L].T * scale
            p = np.exp(x - x.max(axis=1, keepdims=True))
            w = p / p.sum(axis=1, keepdims=True)
            spread[t, rows] = np.einsum("gl,gld->gd", w, np.abs(v[h, None, :L] - O[t, rows][:, None]))
    sums = (length + 64) * 2.0 ** -24 + 2.0 ** -21
    return 1.01 * HALF_STEP["bf16"] * (spread + np.abs(O)) + 1.01 * (2 * Es[..., None] + 2 * sums) * A + 1e-37


@pytest.mark.parametrize("sharp", [1.0, 4.0, 12.0])
def test_rounded_probabilities_cancel_in_prompts(sharp):
    lens = [1, 40, 300, 777]
    T, Hq, Hkv, d = sum(lens), 8, 2, 128
    q, k, v = randn(T, Hq, d, seed=210), randn(T, Hkv, d, seed=211), randn(T, Hkv, d, seed=212)
    k = (k * sharp).to(torch.bfloat16)
    O, lse = run_prefill(q, k, v, lens, "bf16")
    check_prefill(q, k, v, lens, "bf16", O, lse)
    q6, k6, v6, o6 = f64(q), f64(k), f64(v), f64(O)
    at = 0
    for n in lens:
        rows = np.unique(np.linspace(0, n - 1, 40).astype(int))
        ks, vs, vis = k6[at:at + n].swapaxes(0, 1), v6[at:at + n].swapaxes(0, 1), rows + 1
        ref, _, A, Es = attend64(q6[at + rows], ks, vs, vis, d ** -0.5)
        tol = tight_bound(q6[at + rows], ks, vs, vis, d ** -0.5, ref, Es, A, n)
        assert (np.abs(o6[at + rows] - ref) <= tol).all(), f"{n} tokens: {np.max(np.abs(o6[at + rows] - ref) / tol):.2f} of its bound"
        at += n


@pytest.mark.parametrize("new,cached,hint", [([1, 1, 2, 1], [33, 900, 64, 5001], 2), ([40, 17, 64], [200, 5001, 0], 0)])
@pytest.mark.parametrize("sharp", [1.0, 4.0, 12.0])
def test_rounded_probabilities_cancel_over_pages(new, cached, hint, sharp):
    c = PagedCase(new, cached, 8, 2, 128, 64, "bf16", seed=213)
    c.Kp *= sharp
    O, lse = run_paged(c, max_seq=hint)
    q, o = f64(c.Q), f64(O)
    at = 0
    for s, n in enumerate(new):
        rows = np.unique(np.linspace(0, n - 1, 12).astype(int))
        L = cached[s] + n
        k, v, vis = c.slots(c.Kp, s, L), c.slots(c.Vp, s, L), cached[s] + rows + 1
        ref, _, A, Es = attend64(q[at + rows], k, v, vis, 128 ** -0.5)
        tol = tight_bound(q[at + rows], k, v, vis, 128 ** -0.5, ref, Es, A, L)
        assert (np.abs(o[at + rows] - ref) <= tol).all(), f"{n} over {cached[s]}: {np.max(np.abs(o[at + rows] - ref) / tol):.2f} of its bound"
        at += n


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (6, 2, 64), (16, 1, 128)])
@pytest.mark.parametrize("sharp", [1.0, 8.0])
def test_decode_weights_are_good_to_fifteen_bits(Hq, Hkv, d, sharp):
    """A weight's two bf16 parts are off by 2^-15 of it at most, which moves the result by 2^-15 (A + |O|) <= 2^-14 A; what is
    left is the scores' and sums' error and the output's own rounding."""
    new, cached = [1] * 6, [0, 33, 200, 900, 2000, 5001]
    c = PagedCase(new, cached, Hq, Hkv, d, 64, "bf16", seed=218)
    c.Kp *= sharp
    O, lse = run_paged(c, max_seq=1)
    q, o = f64(c.Q), f64(O)
    for s, n in enumerate(cached):
        ref, _, A, Es = attend64(q[s:s + 1], c.slots(c.Kp, s, n + 1), c.slots(c.Vp, s, n + 1), np.array([n + 1]), d ** -0.5)
        sums = (n + 65) * 2.0 ** -24 + 2.0 ** -21
        tol = 1.01 * (HALF_STEP["bf16"] * np.abs(ref) + (2.0 ** -14 + 2 * Es[..., None] + 2 * sums) * A)
        assert (np.abs(o[s:s + 1] - ref) <= tol).all(), f"{n}: {np.max(np.abs(o[s:s + 1] - ref) / tol):.2f} of its bound"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sharp", [1.0, 6.0])
def test_equal_values_come_out_as_they_are(d, sharp):
    """All slots hold one value row: whatever the weights, the result is that row.  Numerator and denominator sum the same
    probabilities in fp32, off by (L + 64) 2^-24 each at most, 1.1e-3 together for L = 9041; half a step of bf16 is 2^-9 =
    1.95e-3 of the value at least, so that rounding lands on the value itself."""
    row = randn(2, d, seed=214)
    lens = [1, 40, 300, 1500]
    T = sum(lens)
    q, k = randn(T, 8, d, seed=215), (randn(T, 2, d, seed=216) * sharp).to(torch.bfloat16)
    v = row[None].expand(T, 2, d).contiguous()
    want = row.repeat_interleave(4, dim=0)
    O, _ = run_prefill(q, k, v, lens, "bf16")
    assert torch.equal(O, want[None].expand_as(O))
    for new, cached, hint in (([1, 1, 2], [1000, 9001, 17], 2), ([40, 64, 5], [9001, 0, 700], 0)):
        c = PagedCase(new, cached, 8, 2, d, 64, "bf16", seed=217)
        c.Kp *= sharp
        c.Vp = row[None, :, None].expand_as(c.Vp).contiguous()
        O, _ = run_paged(c, max_seq=hint)
        assert torch.equal(O, want[None].expand_as(O)), (new, cached)


# ------------------------------------------------------------------------------------------------ references that move
def ramp_case(new, cached, step, big=1.0, seed=220, jitter=0.0):
    """Scores that rise by `step` (in units of log 2) from slot to slot, in element 0 of the keys; scale 1."""
    c = PagedCase(new, cached, 8, 2, 128, 64, "bf16", seed=seed)
    c.Q[..., 0] = math.log(2.0)
    c.Q[..., 1:] *= jitter
    for s, n in enumerate(new):
        for j in range(cached[s] + n):
            c.Kp[int(c.table_cpu[s, j // 64]), :, j % 64, 0] = step * j
    c.Vp *= big
    return c


@pytest.mark.parametrize("new,cached,hint", [([1, 2], [400, 300], 2), ([40, 64], [400, 100], 0)])
def test_large_values_stay_finite_while_scores_rise(new, cached, hint):
    """Values near 2^90 under scores that rise by 2^19 per 128 slots.  A weight is at most 2^16.5 before its reference moves,
    so that every sum stays below 2^16.5 * 500 * 2^93 < 2^119."""
    c = ramp_case(new, cached, 0.15, big=2.0 ** 90)
    O, lse = run_paged(c, max_seq=hint, scale=1.0)
    assert bool(O.isfinite().all())
    check_paged_scaled(c, O, lse)


def check_paged_scaled(c, O, lse):
    q, o, l = f64(c.Q), f64(O), f64(lse)
    at = 0
    for s, n in enumerate(c.new):
        L = c.cached[s] + n
        ref = attend64(q[at:at + n], c.slots(c.Kp, s, L), c.slots(c.Vp, s, L), c.cached[s] + np.arange(1, n + 1), 1.0)
        check_rows(o[at:at + n], l[at:at + n], ref, "bf16", L, f"sequence {s}")
        at += n


@pytest.mark.parametrize("step", [0.05, 0.2, 1.0])
def test_a_moving_reference_repeats_bit_for_bit(step):
    """Rows whose reference moves in one tile after the other, while other groups are at work with the old one."""
    c = ramp_case([40, 128, 300], [700, 2000, 0], step, seed=221, jitter=0.3)
    O, lse = run_paged(c, scale=1.0)
    check_paged_scaled(c, O, lse)
    q, o = f64(c.Q), f64(O)                              # not rounded twice: see tight_bound
    rows = np.arange(40, 168, 9)
    k, v, vis = c.slots(c.Kp, 1, 2128), c.slots(c.Vp, 1, 2128), 2000 + rows - 40 + 1
    ref, _, A, Es = attend64(q[rows], k, v, vis, 1.0)
    assert (np.abs(o[rows] - ref) <= tight_bound(q[rows], k, v, vis, 1.0, ref, Es, A, 2128)).all()
    p = B.Packed(c.Hq, c.Hkv, c.d, c.offsets, c.T, 0, c.dtype)
    h = B.Handle.for_packed(p)
    pages = B.Pages(c.Kp, c.Vp, c.table)
    other = torch.empty((64 << 20,), dtype=torch.uint8, device=DEV)
    for i in range(60):
        O2, lse2 = torch.zeros_like(O), torch.zeros_like(lse)
        if i % 3 == 1:
            other.fill_(i)
        B.samkv_paged_attn(h, p, pages, c.cache_len, c.Q, 1.0, True, O2, lse2)
        assert torch.equal(O, O2) and torch.equal(lse, lse2), f"call {i}"
    assert B.samkv_poll_status(h) == 0


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_positions_pass_31_bits(dtype):
    """Without pages cache_len is only where the positions start: the last of them lie behind 2^31 - 1."""
    c = PagedCase([6, 5], [0, 0], 4, 2, 64, 16, dtype, seed=230)
    p = B.Packed(4, 2, 64, c.offsets, c.T, 0, dtype)
    h = B.Handle.for_packed(p)
    first = [2**31 - 3, 2**31 - 1]
    # turns of 2^-8 to 2^-39 per position: whole numbers of steps, which the 64-bit form counts exactly
    freq = [2.0 * math.pi * 2.0 ** -(8 + i) for i in range(32)]
    K_out, V_out, Q_out = torch.empty_like(c.K), torch.empty_like(c.V), torch.empty_like(c.Q)
    B.samkv_append(h, p, c.K, c.V, None, torch.tensor(first, dtype=torch.int32, device=DEV), B.Rope(64, inv_freq=freq), None,
                   c.Q, Q_out, K_out, V_out)
    assert B.samkv_poll_status(h) == 0
    pos = np.concatenate([first[0] + np.arange(6), first[1] + np.arange(5)]).astype(np.int64)
    turn = np.array([[int(x) % 2 ** (8 + i) / 2.0 ** (8 + i) for i in range(32)] for x in pos])
    for src, got in ((c.K, K_out), (c.Q, Q_out)):
        x = f64(src)
        a, b, cs, sn = x[..., :32], x[..., 32:], np.cos(2 * np.pi * turn)[:, None], np.sin(2 * np.pi * turn)[:, None]
        want = np.concatenate([a * cs - b * sn, b * cs + a * sn], axis=-1)
        # the doubles 2 pi 2^-k are off by 2^-53, and so is the angle: 2^31 * 2 pi 2^-8 * 2^-53 = 1.3e-8 more
        tol = rotate_bound(x, want, 64, False, dtype) + 1.3e-8 * (np.abs(a) + np.abs(b)).repeat(2, axis=-1).max()
        assert (np.abs(f64(got) - want) <= tol).all()
    assert torch.equal(V_out, c.V)


# ------------------------------------------------------------------------------------------------ heights of a row tile
@pytest.mark.parametrize("d,heads,lens", [
    (64, (8, 2), [250, 150]), (128, (8, 2), [250, 150]), (64, (4, 2), [257] * 4),       # 32 rows
    (64, (4, 2), [64] * 7), (64, (4, 2), [33] * 16),                                    # prompts of one key tile: 8 and 32
    (64, (8, 2), [640, 60, 1]), (128, (8, 2), [520]), (64, (4, 2), [1024, 409])])       # 64 rows, at the border
def test_fp32_prompts_of_every_tile_height(d, heads, lens):
    T = sum(lens) + 1
    q, k, v = (randn(T, h, d, dtype="f32", seed=250 + i) for i, h in enumerate((heads[0], heads[1], heads[1])))
    O, lse = run_prefill(q, k, v, lens, "f32")
    check_prefill(q, k, v, lens, "f32", O, lse)


@pytest.mark.parametrize("d,new", [(64, [200, 40, 210]), (64, [64, 70, 300, 20]), (128, [600, 130, 20])])
def test_fp32_chunks_of_tall_tiles(d, new):
    c = PagedCase(new, [100, 0, 513, 64][:len(new)], 8, 2, d, 32, "f32", seed=253, garbage=float("nan"))
    O, lse = run_paged(c)
    check_paged(c, O, lse)


@pytest.mark.parametrize("Hq,Hkv", [(9, 3), (5, 1), (11, 1), (8, 2)])
def test_rows_do_not_depend_on_what_shares_their_tile(Hq, Hkv):
    """Rows of a tile that belong to no token hold whatever an earlier call left there.  Moving references (rising keys)
    between calls that leave other rows behind: bit for bit the same."""
    new, cached = [251, 130, 511], [1679, 588, 943]
    c = PagedCase(new, cached, Hq, Hkv, 128, 64, "bf16", seed=222)
    for s in range(3):
        for j in range(cached[s] + new[s]):
            c.Kp[int(c.table_cpu[s, j // 64]), :, j % 64, 0] += 1.6 * j
    c.Kp *= 4.0
    c.Q[..., 0] = 1.0
    O, lse = run_paged(c)
    other = PagedCase([3000], [0], 8, 2, 128, 64, "bf16", seed=223)          # every row of its tiles is a token
    Q0 = other.Q.clone()
    for i in range(40):
        other.Q = (Q0 * 10.0 ** (i % 5 - 2)).to(torch.bfloat16) if i % 7 else torch.full_like(Q0, float("nan"))
        run_paged(other)
        O2, lse2 = run_paged(c)
        assert torch.equal(O, O2) and torch.equal(lse, lse2), f"call {i}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,cached,hint", [([1, 2, 1], [300, 130, 64], 2), ([40, 9], [300, 20], 0)])
def test_visible_infinities_of_values_come_out(dtype, new, cached, hint):
    """Among slots that all rows see, ones that only some see, and the very last; weights that are powers of two among them
    (equal scores), whose lower bits are zero."""
    for scale in (0.0, 1e-30):                           # (all scores equal: every weight is 1)
        c = PagedCase(new, cached, 8, 2, 128, 64, dtype, seed=260, garbage=float("nan"))
        for s in range(len(new)):
            for j, e, x in ((5, 3, math.inf), (17, 9, -math.inf), (cached[s], 20, math.inf), (cached[s] + new[s] - 1, 127, -math.inf)):
                c.Vp[int(c.table_cpu[s, j // 64]), 1, j % 64, e] = x
        O, lse = run_paged(c, max_seq=hint, scale=scale)
        check_paged(c, O, lse, scale=scale)
