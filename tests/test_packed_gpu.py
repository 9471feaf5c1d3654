"""samkv_prefill, samkv_append and samkv_paged_attn against their plain 64-bit forms (packed_testlib)."""
import math

import numpy as np
import pytest
import torch

from paper_2508_11661_b200 import binding as B
from packed_testlib import DT, PagedCase, attend64, check_rows, f64, rotate64, rotate_bound

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def offsets_of(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV)


def run_prefill(q, k, v, lens, dtype, scale=0.0, want_lse=True, max_seq=0, handle=None, fill=7.0):
    """q [T, Hq, d], k, v [T, Hkv, d] on the GPU (any strides)."""
    T, Hq, d = q.shape
    p = B.Packed(Hq, k.shape[1], d, offsets_of(lens), T, max_seq, dtype)
    h = handle or B.Handle.for_packed(p)
    O = torch.full((T, Hq, d), fill, dtype=q.dtype, device=DEV)
    lse = torch.full((T, Hq), fill, dtype=torch.float32, device=DEV) if want_lse else None
    B.samkv_prefill(h, p, q, k, v, scale, O, lse)
    assert B.samkv_poll_status(h) == 0
    return O, lse


def check_prefill(q, k, v, lens, dtype, O, lse, scale=0.0, fill=7.0):
    scale = scale if scale > 0 else 1.0 / math.sqrt(q.shape[2])
    q6, k6, v6, o6 = f64(q), f64(k), f64(v), f64(O)
    l6 = f64(lse) if lse is not None else None
    at = 0
    for s, n in enumerate(lens):
        r = slice(at, at + n)
        ref = attend64(q6[r], k6[r].swapaxes(0, 1), v6[r].swapaxes(0, 1), np.arange(1, n + 1), scale)
        check_rows(o6[r], None if l6 is None else l6[r], ref, dtype, n, f"sequence {s} of {n}")
        at += n
    assert (o6[at:] == fill).all() and (l6 is None or (l6[at:] == fill).all()), "rows behind the last sequence"


def randn(*shape, dtype="bf16", seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(DT[dtype]).to(DEV)


# ------------------------------------------------------------------------------------------------ prompt attention
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 64), (8, 2, 128), (3, 3, 128), (5, 1, 64), (6, 2, 128), (32, 1, 128)])
def test_prefill_lengths(dtype, Hq, Hkv, d):
    lens = [1, 0, 2, 17, 128, 129, 0, 127, 300, 1, 64, 65, 31, 33, 32]
    T = sum(lens) + 5
    q, k, v = randn(T, Hq, d, dtype=dtype, seed=1), randn(T, Hkv, d, dtype=dtype, seed=2), randn(T, Hkv, d, dtype=dtype, seed=3)
    O, lse = run_prefill(q, k, v, lens, dtype)
    check_prefill(q, k, v, lens, dtype, O, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[1], [5], [700], [1, 1, 1], [0, 9], [513, 255, 257]])
def test_prefill_few_sequences(dtype, lens):
    T = sum(lens)
    q, k, v = randn(T, 8, 128, dtype=dtype, seed=4), randn(T, 2, 128, dtype=dtype, seed=5), randn(T, 2, 128, dtype=dtype, seed=6)
    for max_seq in (0, max(lens), 1):                    # the hint chooses a kernel, never the result
        O, lse = run_prefill(q, k, v, lens, dtype, max_seq=max_seq)
        check_prefill(q, k, v, lens, dtype, O, lse)


def test_prefill_sampled_long_sequence():
    """4000 tokens next to short ones; rows at the tiles' edges and a seeded sample against the 64-bit form."""
    lens = [3, 4000, 130]
    T, Hq, Hkv, d = sum(lens), 8, 2, 128
    q, k, v = randn(T, Hq, d, seed=7), randn(T, Hkv, d, seed=8), randn(T, Hkv, d, seed=9)
    k[:, :, ::32] *= 4.0
    O, lse = run_prefill(q, k, v, lens, "bf16")
    q6, k6, v6, o6, l6 = f64(q), f64(k), f64(v), f64(O), f64(lse)
    rows = sorted(set([0, 1, 31, 32, 127, 128, 129, 2047, 2048, 3999] + list(np.random.default_rng(0).integers(0, 4000, 40))))
    ref = attend64(q6[[3 + r for r in rows]], k6[3:4003].swapaxes(0, 1), v6[3:4003].swapaxes(0, 1),
                   np.array(rows) + 1, d ** -0.5)
    check_rows(o6[[3 + r for r in rows]], l6[[3 + r for r in rows]], ref, "bf16", 4000)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_strides(dtype):
    """Slices of a fused matrix, and the library's [heads, tokens, d] slabs."""
    lens = [40, 200, 7]
    T, Hq, Hkv, d = sum(lens), 8, 2, 128
    fused = randn(T, Hq + 2 * Hkv, d, dtype=dtype, seed=10)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    O, lse = run_prefill(q, k, v, lens, dtype)
    check_prefill(q, k, v, lens, dtype, O, lse)
    slab_k, slab_v = k.permute(1, 0, 2).contiguous(), v.permute(1, 0, 2).contiguous()
    O2, lse2 = run_prefill(q, slab_k.permute(1, 0, 2), slab_v.permute(1, 0, 2), lens, dtype)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    # an output with strides of its own: columns of a wider matrix, whose other columns stay
    p = B.Packed(Hq, Hkv, d, offsets_of(lens), T, 0, dtype)
    h = B.Handle.for_packed(p)
    wide = torch.full((T, Hq + 3, d), 5.0, dtype=DT[dtype], device=DEV)
    B.samkv_prefill(h, p, q, k, v, 0.0, wide[:, 1:1 + Hq])
    assert torch.equal(wide[:, 1:1 + Hq], O) and bool((wide[:, 0] == 5.0).all()) and bool((wide[:, 1 + Hq:] == 5.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["K", "V"])
def test_prefill_values_behind_a_row_do_not_reach_it(dtype, bad, where):
    lens = [150, 300]
    T, Hq, Hkv, d = sum(lens) + 40, 4, 2, 128
    q, k, v = randn(T, Hq, d, dtype=dtype, seed=11), randn(T, Hkv, d, dtype=dtype, seed=12), randn(T, Hkv, d, dtype=dtype, seed=13)
    O, lse = run_prefill(q, k, v, lens, dtype)
    x = (k if where == "K" else v).clone()
    x[150 + 201:, 0, 5] = bad                       # from token 201 of the second sequence on, and the padding rows
    O2, lse2 = run_prefill(q, x if where == "K" else k, x if where == "V" else v, lens, dtype)
    keep = slice(0, 150 + 201)
    assert torch.equal(O[keep], O2[keep]) and torch.equal(lse[keep], lse2[keep])
    assert torch.equal(O[:, 2:], O2[:, 2:])         # the other KV head's queries are untouched
    after = O2[150 + 201:450, :2]
    if where == "V":                                # column 5 carries the value (inf - inf is NaN for none: one sign)
        assert bool((after[..., 5].float() == bad).all()) if bad == bad else bool(after[..., 5].isnan().all())
        assert bool(after[..., 6].isfinite().all())
    elif bad != bad:
        assert bool(after.isnan().all())


def test_prefill_extreme_scores():
    """Scores of thousands, all equal scores, and a scale given by the caller."""
    lens = [260]
    q, k, v = randn(260, 4, 128, seed=14), randn(260, 2, 128, seed=15), randn(260, 2, 128, seed=16)
    for factor, scale in ((64.0, 0.0), (0.0, 0.0), (1.0, 0.5)):
        qq = (q * factor).to(torch.bfloat16)
        O, lse = run_prefill(qq, k, v, lens, "bf16", scale=scale)
        check_prefill(qq, k, v, lens, "bf16", O, lse, scale=scale)
    # keys that grow along the sequence: the running maximum has to follow, far beyond 2^64 in the weights
    ramp = k * torch.arange(260, device=DEV)[:, None, None].to(torch.bfloat16)
    O, lse = run_prefill(q, ramp, v, lens, "bf16", scale=1.0)
    check_prefill(q, ramp, v, lens, "bf16", O, lse, scale=1.0)


# ------------------------------------------------------------------------------------------------ append
def run_append(c: PagedCase, rope=None, positions=None, with_q=True, with_rows=False, handle=None):
    p = B.Packed(c.Hq, c.Hkv, c.d, c.offsets, c.T, 0, c.dtype)
    h = handle or B.Handle.for_packed(p)
    Q_out = torch.full_like(c.Q, 3.0) if with_q else None
    K_out = torch.full_like(c.K, 3.0) if with_rows else None
    V_out = torch.full_like(c.V, 3.0) if with_rows else None
    B.samkv_append(h, p, c.K, c.V, B.Pages(c.Kp, c.Vp, c.table), c.cache_len, rope, positions, c.Q if with_q else None,
                   Q_out, K_out, V_out)
    assert B.samkv_poll_status(h) == 0
    return Q_out, K_out, V_out


def check_append(c: PagedCase, Kp0, Vp0, outs, rot=0, base=1.0, interleaved=False, pos=None, inv_freq=None):
    k, v, q = f64(c.K), f64(c.V), f64(c.Q)
    if pos is None:
        pos = np.concatenate([np.arange(a, a + n) for a, n in zip(c.cached, c.new)] + [np.zeros(c.T - c.total)])
    if rot:
        kr, qr = rotate64(k, pos, rot, base, interleaved, inv_freq), rotate64(q, pos, rot, base, interleaved, inv_freq)
        kt, qt = rotate_bound(k, kr, rot, interleaved, c.dtype), rotate_bound(q, qr, rot, interleaved, c.dtype)
        kt[..., rot:], qt[..., rot:] = 0.0, 0.0
    else:
        kr, qr, kt, qt = k, q, np.zeros_like(k), np.zeros_like(q)
    Kp, Vp = f64(c.Kp), f64(c.Vp)
    eK, eV = f64(Kp0), f64(Vp0)
    tK = np.zeros_like(eK)
    for s, n in enumerate(c.new):
        for t in range(n):
            slot = c.cached[s] + t
            page, r, row = int(c.table_cpu[s, slot // c.page]), slot % c.page, int(c.starts[s]) + t
            eK[page, :, r], eV[page, :, r], tK[page, :, r] = kr[row], v[row], kt[row]
    assert np.array_equal(Vp, eV), "V rows are copied, everything else stays"
    assert (np.abs(Kp - eK) <= tK).all(), f"K pages off by {np.abs(Kp - eK).max():.3e}"
    Q_out, K_out, V_out = outs
    if Q_out is not None:
        got = f64(Q_out)
        assert (np.abs(got - qr)[:c.total] <= qt[:c.total]).all() and (got[c.total:] == 3.0).all()
    if K_out is not None:
        got, gv = f64(K_out), f64(V_out)
        assert (np.abs(got - kr)[:c.total] <= kt[:c.total]).all() and (got[c.total:] == 3.0).all()
        assert np.array_equal(gv[:c.total], v[:c.total]) and (gv[c.total:] == 3.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("rot,interleaved", [(0, False), (128, False), (128, True), (48, False), (48, True), (16, True)])
def test_append(dtype, page, rot, interleaved):
    c = PagedCase([1, 0, 5, 300, 1, 64, 17], [0, 9, page - 1, 33, page, 2 * page - 5, 1000], 6, 2, 128, page, dtype, seed=20, pad=4)
    K0, V0 = c.Kp.clone(), c.Vp.clone()
    rope = B.Rope(rot, 500000.0, interleaved) if rot else None
    outs = run_append(c, rope, with_rows=True)
    check_append(c, K0, V0, outs, rot, 500000.0, interleaved)


@pytest.mark.parametrize("Hq,Hkv,d", [(1, 1, 64), (7, 7, 64), (32, 8, 128), (5, 1, 128)])
def test_append_heads_and_options(Hq, Hkv, d):
    c = PagedCase([3] * 70 + [0, 41], [11] * 70 + [0, 5], Hq, Hkv, d, 16, "bf16", seed=21, pad=1)
    K0, V0 = c.Kp.clone(), c.Vp.clone()
    outs = run_append(c, B.Rope(d, 10000.0), with_q=False)
    check_append(c, K0, V0, outs, d, 10000.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_far_and_negative_positions(dtype):
    c = PagedCase([64, 64], [0, 30], 2, 2, 64, 64, dtype, seed=22)
    K0, V0 = c.Kp.clone(), c.Vp.clone()
    pos = np.concatenate([np.arange(2**31 - 64, 2**31), -np.arange(64) * 1000003])
    t = torch.from_numpy(pos.astype(np.int32)).to(DEV)
    freq = [1.0, 0.3, 6.5, -0.02, 1e-7, 12345.678, 0.5, 2.0 ** -20] * 4
    outs = run_append(c, B.Rope(64, inv_freq=freq), positions=t)
    # the 64-bit form multiplies in long double: at 2^31 radians a double angle is only good to 2^-22
    ang = np.asarray(pos, dtype=np.longdouble)[:, None] * np.asarray(freq, dtype=np.longdouble)[None, :]
    two_pi = np.longdouble(2) * np.longdouble("3.14159265358979323846264338327950288")
    ang = (ang - np.floor(ang / two_pi) * two_pi).astype(np.float64)
    assert np.abs(ang).max() < 6.3
    k = f64(c.K)
    a, b, cs, sn = k[..., :32], k[..., 32:], np.cos(ang)[:, None], np.sin(ang)[:, None]
    want = np.concatenate([a * cs - b * sn, b * cs + a * sn], axis=-1)
    # 12345.678 * 2^31 = 2.7e13 radians: the long double product is good to 2^-64 of that, 1.4e-6
    tol = rotate_bound(k, want, 64, False, dtype) + 1.5e-6 * (np.abs(a) + np.abs(b)).repeat(2, axis=-1).max()
    got = np.concatenate([c_ for c_ in [np.swapaxes(c.slots(c.Kp, 0, 64), 0, 1), np.swapaxes(c.slots(c.Kp, 1, 94), 0, 1)[30:]]])
    assert (np.abs(got - want) <= tol).all()


def test_append_in_place_and_rows_only():
    c = PagedCase([50, 3], [0, 0], 8, 2, 128, 64, "bf16", seed=23)
    p = B.Packed(8, 2, 128, c.offsets, c.T, 0, "bf16")
    h = B.Handle.for_packed(p)
    rope = B.Rope(128, 10000.0)
    Q1, K1, V1 = torch.empty_like(c.Q), torch.empty_like(c.K), torch.empty_like(c.V)
    B.samkv_append(h, p, c.K, c.V, None, None, rope, None, c.Q, Q1, K1, V1)
    slab = torch.empty((2, c.T, 128), dtype=torch.bfloat16, device=DEV)     # the [heads, tokens, d] layout of a document cache
    V2 = torch.empty_like(c.V)
    B.samkv_append(h, p, c.K, c.V, None, None, rope, None, None, None, slab.permute(1, 0, 2), V2)
    q, k, v = c.Q.clone(), c.K.clone(), c.V.clone()
    B.samkv_append(h, p, k, v, None, None, rope, None, q, q, k, v)          # in place
    assert B.samkv_poll_status(h) == 0
    assert torch.equal(q, Q1) and torch.equal(k, K1) and torch.equal(v, c.V) and torch.equal(V1, c.V) and torch.equal(V2, c.V)
    assert torch.equal(slab.permute(1, 0, 2), K1)


def test_append_bad_pages_and_full_tables_are_reported_and_skipped():
    c = PagedCase([4, 40], [14, 0], 2, 2, 64, 16, "bf16", seed=24, spare_cols=0)
    p = B.Packed(2, 2, 64, c.offsets, c.T, 0, "bf16")
    h = B.Handle.for_packed(p)
    table = c.table.clone()
    table[0, 1], table[1, 2] = -3, c.n_pages
    K0, V0 = c.Kp.clone(), c.Vp.clone()
    B.samkv_append(h, p, c.K, c.V, B.Pages(c.Kp, c.Vp, table), c.cache_len)
    assert B.samkv_poll_status(h) == 7 and B.samkv_poll_status(h) == 0
    changed = (c.Kp != K0).flatten(1).any(1).nonzero().flatten().tolist()
    assert set(changed) <= {int(table[0, 0]), int(table[1, 0]), int(table[1, 1])}
    # lengths behind the table's end
    c.Kp.copy_(K0)
    c.Vp.copy_(V0)
    B.samkv_append(h, p, c.K, c.V, B.Pages(c.Kp, c.Vp, c.table), torch.tensor([2**31 - 2, 16 * c.width], dtype=torch.int32, device=DEV))
    assert B.samkv_poll_status(h) == 7
    assert torch.equal(c.Kp, K0) and torch.equal(c.Vp, V0)
    # offsets that leave the packed rows, or run backwards
    off = torch.tensor([-5, 20, 2**30], dtype=torch.int32, device=DEV)
    p2 = B.Packed(2, 2, 64, off, c.T, 0, "bf16")
    B.samkv_append(h, p2, c.K, c.V, B.Pages(c.Kp, c.Vp, c.table), torch.zeros(2, dtype=torch.int32, device=DEV))
    assert B.samkv_poll_status(h) == 7


# ------------------------------------------------------------------------------------------------ paged attention
def run_paged(c: PagedCase, causal=True, scale=0.0, max_seq=0, handle=None, fill=7.0, poll=0):
    p = B.Packed(c.Hq, c.Hkv, c.d, c.offsets, c.T, max_seq, c.dtype)
    h = handle or B.Handle.for_packed(p)
    O = torch.full_like(c.Q, fill)
    lse = torch.full((c.T, c.Hq), fill, dtype=torch.float32, device=DEV)
    B.samkv_paged_attn(h, p, B.Pages(c.Kp, c.Vp, c.table), c.cache_len, c.Q, scale, causal, O, lse)
    assert B.samkv_poll_status(h) == poll
    return O, lse


def check_paged(c: PagedCase, O, lse, causal=True, scale=0.0, fill=7.0):
    scale = scale if scale > 0 else 1.0 / math.sqrt(c.d)
    q, o, l = f64(c.Q), f64(O), f64(lse)
    at = 0
    for s, n in enumerate(c.new):
        length = c.cached[s] + (n if causal else 0)
        vis = c.cached[s] + (np.arange(1, n + 1) if causal else np.zeros(n, dtype=int))
        k, v = c.slots(c.Kp, s, length), c.slots(c.Vp, s, length)
        r = slice(at, at + n)
        check_rows(o[r], l[r], attend64(q[r], k, v, vis, scale), c.dtype, length, f"sequence {s}: {n} over {c.cached[s]}")
        at += n
    assert (o[at:] == fill).all() and (l[at:] == fill).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (4, 2, 64), (3, 3, 128), (32, 1, 64)])
def test_decode(dtype, page, Hq, Hkv, d):
    """One token per sequence; unused slots of the last page hold NaN."""
    cached = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 500, 0, 1000, 333]
    c = PagedCase([1] * len(cached), cached, Hq, Hkv, d, page, dtype, seed=30, garbage=float("nan"))
    O, lse = run_paged(c, max_seq=1)
    check_paged(c, O, lse)
    O2, lse2 = run_paged(c, max_seq=0)
    check_paged(c, O2, lse2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (4, 2, 64), (5, 1, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_chunks(dtype, page, Hq, Hkv, d, causal):
    """Chunks and single tokens mixed; without the causal tail a sequence with an empty cache has empty rows."""
    c = PagedCase([1, 5, 0, 64, 130, 1, 33, 7], [300, 0, 20, 131, 77, 0, 640, 16], Hq, Hkv, d, page, dtype, seed=31, pad=3,
                  garbage=float("nan"))
    O, lse = run_paged(c, causal)
    check_paged(c, O, lse, causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,Hq,Hkv", [(1, 8, 1), (1, 8, 8), (4, 16, 2), (40, 8, 2)])
def test_long_cache_is_split(dtype, new, Hq, Hkv):
    """One sequence over a long cache: the keys are divided among the CTAs and merged.  Twice, bit for bit."""
    c = PagedCase([new], [9001], Hq, Hkv, 128, 64, dtype, seed=32)
    O, lse = run_paged(c)
    check_paged(c, O, lse)
    O2, lse2 = run_paged(c)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)


def test_many_sequences():
    """More sequences than one pass of a block covers, most of them one token long."""
    r = np.random.default_rng(5)
    new = [1] * 1500 + [int(x) for x in r.integers(0, 4, 500)]
    cached = [int(x) for x in r.integers(0, 40, 2000)]
    c = PagedCase(new, cached, 4, 2, 64, 16, "bf16", seed=33)
    O, lse = run_paged(c, max_seq=3)
    check_paged(c, O, lse)


@pytest.mark.parametrize("new", [1, 20])
def test_bad_pages_are_reported(new):
    c = PagedCase([new, new], [100, 50], 4, 2, 128, 16, "bf16", seed=34)
    good, lse = run_paged(c)
    c.table[0, 2] = c.n_pages + 7
    O, lse = run_paged(c, poll=7)
    assert torch.equal(O[new:], good[new:])                     # the other sequence is what it was
    c.table[0, 2] = -1
    O, lse = run_paged(c, poll=7)
    c.table[0, 2] = c.table_cpu[0, 2]
    O, lse = run_paged(c)
    assert torch.equal(O, good)
    # a cache length behind the table's end is cut off and reported
    p = B.Packed(4, 2, 128, c.offsets, c.T, 0, "bf16")
    h = B.Handle.for_packed(p)
    full = c.table.clamp(min=0)
    B.samkv_paged_attn(h, p, B.Pages(c.Kp, c.Vp, full.contiguous()),
                       torch.tensor([2**31 - 1, -4], dtype=torch.int32, device=DEV), c.Q, 0.0, True, O)
    assert B.samkv_poll_status(h) == 7


def test_extreme_values():
    c = PagedCase([1, 9], [200, 300], 4, 2, 128, 64, "bf16", seed=35)
    c.Kp *= 40.0
    for causal in (True, False):
        O, lse = run_paged(c, causal)
        check_paged(c, O, lse, causal)
    # keys that grow along the cache by far more than a weight's range
    c = PagedCase([3, 40], [900, 700], 4, 2, 128, 64, "bf16", seed=36)
    for s in range(2):
        for j in range(c.cached[s] + c.new[s]):
            c.Kp[int(c.table_cpu[s, j // 64]), :, j % 64] *= j
    O, lse = run_paged(c, scale=1.0)
    check_paged(c, O, lse, scale=1.0)
    # a visible NaN key or value reaches exactly the rows that see it
    c = PagedCase([6, 40], [70, 10], 4, 2, 128, 64, "bf16", seed=37)
    for s, j in ((0, 72), (1, 30)):
        c.Vp[int(c.table_cpu[s, j // 64]), 1, j % 64, 9] = float("nan")
        c.Kp[int(c.table_cpu[s, (j + 2) // 64]), 0, (j + 2) % 64, 100] = float("nan")
    O, lse = run_paged(c)
    check_paged(c, O, lse)


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_then_decode_through_pages_equals_one_prompt(dtype):
    """Append + attend in chunks of changing size gives what one causal pass over the whole prompt gives."""
    Hq, Hkv, d, page = 8, 2, 128, 16
    total = [70, 33, 150]
    T = sum(total)
    q, k, v = randn(T, Hq, d, dtype=dtype, seed=40), randn(T, Hkv, d, dtype=dtype, seed=41), randn(T, Hkv, d, dtype=dtype, seed=42)
    off = np.concatenate([[0], np.cumsum(total)])
    rope = B.Rope(128, 10000.0)
    whole = B.Packed(Hq, Hkv, d, offsets_of(total), T, 0, dtype)
    h = B.Handle.for_packed(whole)
    qr, kr, vr = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    B.samkv_append(h, whole, k, v, None, None, rope, None, q, qr, kr, vr)
    O1, lse1 = torch.empty_like(q), torch.empty((T, Hq), dtype=torch.float32, device=DEV)
    B.samkv_prefill(h, whole, qr, kr, vr, 0.0, O1, lse1)
    check_prefill(qr, kr, vr, total, dtype, O1, lse1)
    width = 10
    Kp = torch.zeros((40, Hkv, page, d), dtype=DT[dtype], device=DEV)
    pages = B.Pages(Kp, torch.zeros_like(Kp), torch.randperm(40)[:30].to(torch.int32).view(3, 10).contiguous().to(DEV))
    done = [0, 0, 0]
    O2, lse2 = torch.zeros_like(O1), torch.zeros_like(lse1)
    steps = [[20, 0, 64], [1, 1, 1], [30, 5, 17], [1, 1, 1], [18, 26, 67]]
    for step in steps:
        idx = np.concatenate([np.arange(off[s] + done[s], off[s] + done[s] + n) for s, n in enumerate(step)])
        idx = torch.from_numpy(idx).to(DEV)
        p = B.Packed(Hq, Hkv, d, offsets_of(step), sum(step), max(step), dtype)
        lens = torch.tensor(done, dtype=torch.int32, device=DEV)
        qs = torch.empty((sum(step), Hq, d), dtype=DT[dtype], device=DEV)
        B.samkv_append(h, p, k[idx].contiguous(), v[idx].contiguous(), pages, lens, rope, None, q[idx].contiguous(), qs)
        o, l = torch.empty_like(qs), torch.empty((sum(step), Hq), dtype=torch.float32, device=DEV)
        B.samkv_paged_attn(h, p, pages, lens, qs, 0.0, True, o, l)
        O2[idx], lse2[idx] = o, l
        done = [a + b for a, b in zip(done, step)]
    assert done == total and B.samkv_poll_status(h) == 0
    check_prefill(qr, kr, vr, total, dtype, O2, lse2)


def test_documents_prefilled_into_the_cache_that_scoring_and_compaction_read():
    """The serving path around the sparsified cache: the projections of packed documents are rotated into the library's
    own slabs (samkv_append), attended (samkv_prefill), scored and compacted, and the query attends over what is kept."""
    from paper_2508_11661_b200 import synth
    import samkv_testlib as T
    w = synth.CONFIGS["cfg1"].replace(ctx_lens=(257, 64, 500), n_q_heads=8, n_kv_heads=2)
    inp = {n: t.to(DEV) for n, t in synth.make_inputs(w, "cpu").items()}
    L = w.l_tot
    raw_k, raw_v, raw_q = randn(L, 2, 128, seed=50), randn(L, 2, 128, seed=51), randn(L, 8, 128, seed=52)
    p = B.Packed(8, 2, 128, torch.tensor(w.ctx_offsets, dtype=torch.int32, device=DEV), L)
    h = B.Handle.for_packed(p)
    q = torch.empty_like(raw_q)
    K, V = inp["K"][0, 0], inp["V"][0, 0]                          # [Hkv, L_tot, d]
    B.samkv_append(h, p, raw_k, raw_v, None, None, B.Rope(128, w.rope_base), None, raw_q, q, K.permute(1, 0, 2), V.permute(1, 0, 2))
    O = torch.empty_like(q)
    B.samkv_prefill(h, p, q, K.permute(1, 0, 2), V.permute(1, 0, 2), 0.0, O)
    assert B.samkv_poll_status(h) == 0
    pos = np.concatenate([np.arange(n) for n in w.ctx_lens])
    want = rotate64(f64(raw_k), pos, 128, w.rope_base, False)
    assert (np.abs(np.swapaxes(f64(K), 0, 1) - want) <= rotate_bound(f64(raw_k), want, 128, False, "bf16")).all()
    check_prefill(q, K.permute(1, 0, 2), V.permute(1, 0, 2), list(w.ctx_lens), "bf16", O, None)
    run = T.DeviceRun(w, inp).sparsify()
    torch.cuda.synchronize()
    qh, _, u = T.oracle_scores(w, inp, 0, 0)
    sel = run.sel.cpu().numpy()
    T.check_scores(w, run, 0, 0, qh, u)
    T.check_selection(w, run.k_units, sel[0, 0], u)
    T.check_compact(w, run, 0, 0, sel[0, 0])
    Kc, Vc = run.Kc[0, 0].clone(), run.Vc[0, 0].clone()
    Og, lse = run.attn(0, inp["Qa"][0], inp["Kq"][0], inp["Vq"][0])
    torch.cuda.synchronize()
    T.check_attention(w, Kc, Vc, run.S, inp["Qa"][0, 0], inp["Kq"][0, 0], inp["Vq"][0, 0], Og[0], lse[0])
    assert run.poll() == 0


# ------------------------------------------------------------------------------------------------ streams and graphs
@pytest.mark.parametrize("new", [1, 24])
def test_captured_step_replays_with_new_lengths(new):
    """Append and attention captured once, replayed while the lengths grow and the inputs change; on a side stream."""
    c = PagedCase([new] * 3, [30, 0, 200], 8, 2, 128, 64, "bf16", seed=60, spare_cols=4)
    c.table.copy_(torch.arange(3 * c.width, dtype=torch.int32).view(3, -1))
    Kp = torch.zeros((3 * c.width, 2, 64, 128), dtype=torch.bfloat16, device=DEV)
    pages = B.Pages(Kp, torch.zeros_like(Kp), c.table)
    p = B.Packed(8, 2, 128, c.offsets, c.T, new)
    rope = B.Rope(128, 10000.0)

    def fresh():
        return B.Handle.for_packed(p), torch.empty_like(c.Q), torch.empty_like(c.Q)

    h, qs, O = fresh()
    lens = c.cache_len.clone()
    K, V, Q = c.K.clone(), c.V.clone(), c.Q.clone()

    def step(h, K, V, Q, qs, O, lens, pages):
        B.samkv_append(h, p, K, V, pages, lens, rope, None, Q, qs)
        B.samkv_paged_attn(h, p, pages, lens, qs, 0.0, True, O)
        lens += new

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step(h, K, V, Q, qs, O, lens, pages)              # warm-up outside the capture
        lens.copy_(c.cache_len)
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            step(h, K, V, Q, qs, O, lens, pages)
    Kp.zero_()
    pages.V.zero_()
    lens.copy_(c.cache_len)
    h2, qs2, O2 = fresh()
    lens2 = c.cache_len.clone()
    pages2 = B.Pages(torch.zeros_like(Kp), torch.zeros_like(Kp), c.table)
    for i in range(6):
        for t, seed in ((K, 1), (V, 2), (Q, 3)):
            t.copy_(randn(*t.shape, seed=100 * i + seed))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        step(h2, K, V, Q, qs2, O2, lens2, pages2)
        torch.cuda.synchronize()
        assert torch.equal(O, O2) and torch.equal(lens, lens2) and torch.equal(Kp, pages2.K), f"replay {i}"
    assert B.samkv_poll_status(h) == 0


@pytest.mark.parametrize("new", [1, 40])
def test_stream_order_on_every_input(new):
    """Kernels that write Q, the pages and the lengths directly before each call must be seen by it."""
    c = PagedCase([new, new], [700, 120], 8, 2, 128, 64, "bf16", seed=61)
    p = B.Packed(8, 2, 128, c.offsets, c.T, new)
    h = B.Handle.for_packed(p)
    pages = B.Pages(c.Kp, c.Vp, c.table)
    ref, outs = [], []
    Q0, K0 = c.Q.clone(), c.Kp.clone()
    for i in range(24):
        c.Q.copy_(Q0 * (1.0 - 0.03 * i))
        c.Kp.copy_(K0 * (1.0 + 0.01 * i))
        c.cache_len.fill_(100 + i)
        O = torch.empty_like(c.Q)
        B.samkv_paged_attn(h, p, pages, c.cache_len, c.Q, 0.0, True, O)
        outs.append(O)
    torch.cuda.synchronize()
    for i in range(24):
        c.Q.copy_(Q0 * (1.0 - 0.03 * i))
        c.Kp.copy_(K0 * (1.0 + 0.01 * i))
        c.cache_len.fill_(100 + i)
        torch.cuda.synchronize()
        O = torch.empty_like(c.Q)
        B.samkv_paged_attn(h, p, pages, c.cache_len, c.Q, 0.0, True, O)
        torch.cuda.synchronize()
        assert torch.equal(O, outs[i]), f"call {i}"
    assert B.samkv_poll_status(h) == 0


def test_workspace_and_handle_refusals():
    c = PagedCase([4], [10], 8, 2, 128, 64, "bf16", seed=62)
    p = B.Packed(8, 2, 128, c.offsets, c.T)
    O = torch.empty_like(c.Q)
    need = B.samkv_packed_workspace_bytes(p)
    if need > 4096:
        h = B.Handle.for_packed(p)
        small = torch.empty(need - 256, dtype=torch.uint8, device=DEV)
        import ctypes
        raw = ctypes.c_void_p()
        assert B.lib().samkv_create(ctypes.byref(raw), 0, small.data_ptr(), need - 256) == 0
        assert B.lib().samkv_paged_attn(raw, p.ref(), B.Pages(c.Kp, c.Vp, c.table).checked(p), c.cache_len.data_ptr(),
                                        p.rows(c.Q, (c.T, 8, 128), "Q", 0), 0.0, 1, p.rows(O, (c.T, 8, 128), "O", 0), None,
                                        None) == 3
        torch.cuda.synchronize()
        B.lib().samkv_destroy(raw)
    # nothing to do
    p0 = B.Packed(8, 2, 128, c.offsets, 0)
    h = B.Handle.for_packed(p0)
    e = c.Q[:0]
    B.samkv_prefill(h, p0, e, c.K[:0], c.V[:0], 0.0, O[:0])
    B.samkv_append(h, p0, c.K[:0], c.V[:0], B.Pages(c.Kp, c.Vp, c.table), c.cache_len)
    B.samkv_paged_attn(h, p0, B.Pages(c.Kp, c.Vp, c.table), c.cache_len, e, 0.0, True, O[:0])
    assert B.samkv_poll_status(h) == 0
    with pytest.raises(ValueError):
        B.samkv_paged_attn(h, p, B.Pages(c.Kp, c.Vp, c.table), c.cache_len, c.Q.float(), 0.0, True, O)
    with pytest.raises(ValueError):
        B.samkv_paged_attn(h, p, B.Pages(c.Kp, c.Vp, c.table), c.cache_len.long(), c.Q, 0.0, True, O)


def test_chunks_over_keys_that_l2_cannot_hold():
    """Several row tiles over more than 64 MB of keys run in waves of equal blocks; rows at the tiles' edges against the
    64-bit form, the others against the contiguous layout of the same work (one KV head at a time), and twice bit for bit."""
    for new, cached, Hq, Hkv in (([70, 1, 33], [60000, 300, 9000], 16, 2), ([300], [70001], 8, 2)):
        c = PagedCase(new, cached, Hq, Hkv, 128, 64, "bf16", seed=63)
        O, lse = run_paged(c)
        O2, lse2 = run_paged(c)
        assert torch.equal(O, O2) and torch.equal(lse, lse2)
        q, o, l = f64(c.Q), f64(O), f64(lse)
        at = 0
        for s, n in enumerate(new):
            length = cached[s] + n
            rows = sorted({0, n // 2, n - 1, min(15, n - 1), min(16, n - 1)})
            k, v = c.slots(c.Kp, s, length), c.slots(c.Vp, s, length)
            ref = attend64(q[[at + r for r in rows]], k, v, cached[s] + np.array(rows) + 1, 128 ** -0.5)
            check_rows(o[[at + r for r in rows]], l[[at + r for r in rows]], ref, "bf16", length, f"sequence {s}")
            at += n
        G = Hq // Hkv
        one = PagedCase(new, cached, G, 1, 128, 64, "bf16", seed=63)
        for h in range(Hkv):
            one.Q = c.Q[:, h * G:(h + 1) * G].contiguous()
            one.table = c.table
            one.Kp, one.Vp = c.Kp[:, h:h + 1].contiguous(), c.Vp[:, h:h + 1].contiguous()
            O1, lse1 = run_paged(one)
            # both round the probabilities to 8 bits against other references: each is within its bound of the exact one
            big = O1.abs().amax().float()
            assert bool(((O1 - O[:, h * G:(h + 1) * G]).float().abs() <= 2.0 ** -6 * big).all())
            assert bool((lse1 - lse[:, h * G:(h + 1) * G]).abs().le(1e-4).all())


def test_waves_with_a_sequence_that_sees_nothing():
    """The layout in waves (see above) next to a sequence without cached tokens and no causal tail: its rows are empty."""
    c = PagedCase([300, 5, 0], [70001, 0, 12], 8, 2, 128, 64, "bf16", seed=64)
    O, lse = run_paged(c, causal=False)
    assert bool((O[300:] == 0).all()) and bool((lse[300:] == -math.inf).all())
    q, k, v = f64(c.Q)[:2], c.slots(c.Kp, 0, 70001), c.slots(c.Vp, 0, 70001)
    check_rows(f64(O)[:2], f64(lse)[:2], attend64(q, k, v, [70001, 70001], 128 ** -0.5), "bf16", 70001)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_hint_never_changes_what_is_computed(dtype):
    c = PagedCase([40, 1, 9], [100, 33, 5000], 8, 2, 128, 32, dtype, seed=65)
    for hint in (0, 1, 3, 40, 1000):
        O, lse = run_paged(c, max_seq=hint)
        check_paged(c, O, lse)


def test_first_call_of_a_fresh_handle_on_a_side_stream():
    """Split work right after the handle was made, on a stream that the default stream does not order."""
    c = PagedCase([1], [9001], 8, 1, 128, 64, "bf16", seed=66)
    ref, _ = run_paged(c)
    junk = [torch.full((8 << 20,), 255, dtype=torch.uint8, device=DEV) for _ in range(8)]
    torch.cuda.synchronize()
    del junk                                             # whatever the allocator hands out next is not zero
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        O, _ = run_paged(c)
    torch.cuda.synchronize()
    assert torch.equal(O, ref)


def test_overlapping_offsets_and_foreign_rows_are_reported():
    """Offsets that run backwards are clamped and reported; rows before the first sequence are not touched."""
    c = PagedCase([10, 20], [64, 64], 4, 2, 64, 16, "bf16", seed=67)
    p = B.Packed(4, 2, 64, torch.tensor([6, 10, 8], dtype=torch.int32, device=DEV), c.T)
    h = B.Handle.for_packed(p)
    O = torch.full_like(c.Q, 7.0)
    B.samkv_paged_attn(h, p, B.Pages(c.Kp, c.Vp, c.table), c.cache_len, c.Q, 0.0, True, O)
    assert B.samkv_poll_status(h) == 7
    assert bool((O[:6] == 7.0).all()) and bool((O[10:] == 7.0).all()) and not bool((O[6:10] == 7.0).any())
    B.samkv_paged_attn(h, p, B.Pages(c.Kp, c.Vp, c.table), c.cache_len, c.Q, 0.0, True, O)
    assert B.samkv_poll_status(h) == 7 and B.samkv_poll_status(h) == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[100, 50, 61, 90, 1], [40, 48, 33, 47], [700, 3, 515], [9, 4, 17, 2, 30], [640, 1000]])
def test_fp32_row_tiles(d, lens):
    """The fp32 kernel's heights of a row tile (8, 32, 64 rows, by the rows of the call and their lengths), and what a row does
    not see: infinities and NaN behind it change no bit."""
    T, Hq, Hkv = sum(lens) + 3, 8, 2
    q, k, v = (randn(T, h, d, dtype="f32", seed=70 + i) for i, h in enumerate((Hq, Hkv, Hkv)))
    O, lse = run_prefill(q, k, v, lens, "f32")
    check_prefill(q, k, v, lens, "f32", O, lse)
    at = lens[0] + lens[1] // 2 + 1                      # in the second sequence, seldom on a tile's border
    for bad in (float("nan"), float("inf"), -float("inf")):
        k2, v2 = k.clone(), v.clone()
        k2[at:sum(lens[:2])], v2[at:sum(lens[:2])] = bad, bad
        O2, lse2 = run_prefill(q, k2, v2, lens, "f32")
        keep = torch.ones(T, dtype=torch.bool, device=DEV)
        keep[at:sum(lens[:2])] = False
        assert torch.equal(O[keep], O2[keep]) and torch.equal(lse[keep], lse2[keep])


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 64), (8, 2, 128), (32, 1, 64), (11, 1, 128), (14, 2, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_fp32_tall_row_tiles_over_pages(Hq, Hkv, d, causal):
    c = PagedCase([700, 0, 3, 515], [0, 10, 300, 77], Hq, Hkv, d, 16, "f32", seed=73, pad=2, garbage=float("nan"))
    O, lse = run_paged(c, causal)
    check_paged(c, O, lse, causal)
    O2, lse2 = run_paged(c, causal)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
