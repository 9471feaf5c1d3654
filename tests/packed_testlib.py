"""Plain 64-bit forms of the packed and paged operators, and the bounds their tests use.

Bounds (per output element; A = sum_j w_j |v_j| is the result's size before cancellation):
  scores        a product of d terms summed in fp32 is off by at most (d + 2) 2^-24 sum_i |q_i k_i|, times the scale: E_s
  weights       exp of a score that is off by E_s, the fp32 exponential (2^-22), and for bf16 the rounding of the
                probability to 8 bits (half a step: 2^-8 relative)
  sums          fp32, at most (L + 64) additions and rescalings of 2^-24 each
  result        numerator and denominator each carry the weights' error: 2 E_s + sums, plus half a step of the result's type
  lse           E_s + sums + half a step of fp32 of the value
A NaN or infinity must come out as in the 64-bit form."""
from __future__ import annotations

import numpy as np
import torch

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def attend64(q, k, v, vis, scale):
    """q [n, Hq, d], k, v [Hkv, L, d] (float64), vis [n]: row t sees keys 0 .. vis[t]-1.
    Returns O, lse, A, E_s (E_s: the score bound's 2^-24 factor included)."""
    n, Hq, d = q.shape
    G = Hq // k.shape[0]
    O, A = np.zeros_like(q), np.zeros_like(q)
    lse, Es = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    for t in range(n):
        L = int(vis[t])
        if L <= 0:
            continue
        for h in range(k.shape[0]):
            kk, vv = k[h, :L], v[h, :L]
            rows = slice(h * G, (h + 1) * G)
            with np.errstate(invalid="ignore", over="ignore"):
                x = q[t, rows] @ kk.T * scale                           # [G, L]
                m = x.max(axis=1, keepdims=True)
                p = np.exp(x - m)
                l = p.sum(axis=1, keepdims=True)
                w = p / l
                O[t, rows] = w @ vv
                A[t, rows] = w @ np.abs(vv)
                lse[t, rows] = (m + np.log(l))[:, 0]
                Es[t, rows] = ((d + 2) * 2.0 ** -24 * (np.abs(q[t, rows]) @ np.abs(kk).T)).max(axis=1) * abs(scale)
    return O, lse, A, Es


def check_rows(got_o, got_lse, ref, dtype, length, where=""):
    """got_o [n, Hq, d], got_lse [n, Hq] (numpy float64) against attend64's output."""
    O, lse, A, Es = ref
    sums = (length + 64) * 2.0 ** -24 + 2.0 ** -21
    p_round = HALF_STEP["bf16"] if dtype == "bf16" else 0.0
    tol = (2 * Es[..., None] + 2 * sums + p_round) * 1.01 * A + HALF_STEP[dtype] * 1.01 * np.abs(O) + 1e-37
    assert np.array_equal(np.isnan(O), np.isnan(got_o)), f"{where}: NaN in other places"
    fine = np.isfinite(O)
    assert np.array_equal(O[~fine & ~np.isnan(O)], got_o[~fine & ~np.isnan(O)]), f"{where}: infinities differ"
    err = np.abs(got_o[fine] - O[fine]) - tol[fine]
    assert err.size == 0 or err.max() <= 0, f"{where}: output off by {np.abs(got_o[fine] - O[fine]).max():.3e} ({err.max():.3e} over its bound)"
    if got_lse is not None:
        assert np.array_equal(np.isneginf(lse), np.isneginf(got_lse)), f"{where}: empty rows differ"
        assert np.array_equal(np.isnan(lse), np.isnan(got_lse)), f"{where}: NaN lse in other places"
        ok = np.isfinite(lse)
        t2 = Es[ok] + sums + 2.0 ** -23 * np.abs(lse[ok])
        assert (np.abs(got_lse[ok] - lse[ok]) <= t2).all(), f"{where}: lse off by {np.abs(got_lse[ok] - lse[ok]).max():.3e}"


def rotate64(x, pos, rot, base, interleaved, inv_freq=None):
    """x [n, H, d] float64, pos [n]."""
    half = rot // 2
    f = np.asarray(inv_freq, dtype=np.float64) if inv_freq is not None else float(base) ** (-np.arange(half) / half)
    ang = np.asarray(pos, dtype=np.float64)[:, None] * f[None, :]
    c, s = np.cos(ang)[:, None, :], np.sin(ang)[:, None, :]
    y = x.copy()
    i0, i1 = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
    a, b = x[..., i0], x[..., i1]
    y[..., i0], y[..., i1] = a * c - b * s, b * c + a * s
    return y


def rotate_bound(x, y, rot, interleaved, dtype):
    """Half a step of the type, the fp32 products (2^-24 each, three of them) and a sine or cosine good to 2^-23: every
    element is built from its pair, so the pair's size carries the error."""
    half = rot // 2
    pair = np.zeros_like(x)
    i0, i1 = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
    size = np.abs(x[..., i0]) + np.abs(x[..., i1])
    pair[..., i0], pair[..., i1] = size, size
    return HALF_STEP[dtype] * 1.01 * np.abs(y) + 4 * 2.0 ** -23 * pair + 1e-37


class PagedCase:
    """Seeded tensors of a paged cache: pools, a shuffled table with -1 in unused entries, packed offsets."""

    def __init__(self, new, cached, Hq, Hkv, d, page, dtype, seed=0, pad=0, dev="cuda", garbage=None, spare_cols=2):
        g = torch.Generator().manual_seed(seed)
        self.new, self.cached = list(new), list(cached)
        self.Hq, self.Hkv, self.d, self.page, self.dtype, self.dev = Hq, Hkv, d, page, dtype, dev
        self.T = sum(new) + pad
        self.total = sum(new)
        off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.starts = off
        self.offsets = torch.from_numpy(off).to(dev)
        need = [-(-(c + n) // page) for c, n in zip(cached, new)]
        self.width = max(max(need), 1) + spare_cols
        self.n_pages = sum(need) + 3
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        table = torch.full((len(new), self.width), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = order[at:at + n]
            at += n
        self.table_cpu = table
        self.table = table.to(dev)
        self.cache_len = torch.tensor(self.cached, dtype=torch.int32, device=dev)
        dt = DT[dtype]
        self.Kp = torch.randn((self.n_pages, Hkv, page, d), generator=g).to(dt)
        self.Vp = torch.randn((self.n_pages, Hkv, page, d), generator=g).to(dt)
        self.Q = torch.randn((self.T, Hq, d), generator=g).to(dt)
        self.K = torch.randn((self.T, Hkv, d), generator=g).to(dt)
        self.V = torch.randn((self.T, Hkv, d), generator=g).to(dt)
        if garbage is not None:                       # every slot no sequence owns
            owned = torch.zeros((self.n_pages, page), dtype=torch.bool)
            for s in range(len(new)):
                for j in range(cached[s] + new[s]):
                    owned[table[s, j // page], j % page] = True
            self.Kp[(~owned)[:, None, :].expand(-1, Hkv, -1)] = garbage
            self.Vp[(~owned)[:, None, :].expand(-1, Hkv, -1)] = garbage
        for name in ("Kp", "Vp", "Q", "K", "V"):
            setattr(self, name, getattr(self, name).to(dev))

    def slots(self, pool, s, length):
        """[Hkv, length, d] float64 of sequence s, through the table."""
        n = -(-length // self.page)
        x = f64(pool)[self.table_cpu[s, :n].numpy()]
        return np.swapaxes(x, 0, 1).reshape(self.Hkv, n * self.page, self.d)[:, :length]
