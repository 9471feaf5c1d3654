"""Plain 64-bit form of attention with modified scores, and the bounds its tests use.

Bounds, first order in the error e_j of the score of slot j (w: the weights, A = sum_j w_j |v_j|):
  product      d terms summed in fp32: (d + 2) 2^-24 scale sum_i |q_i k_i|
  cap          has slope <= 1, so that the product's error does not grow; the kernels' own tanh is good to 2^-20 of the value
  distance     slope * |p - j| from a tile's border on: 4 roundings of 2^-24 of |x| + |bias| + 128 |slope| in all
  output       sum_j w_j |v_j| e_j + A sum_j w_j e_j, plus what packed_testlib counts: sums, the rounding of the weights to bf16
               where the output is bf16, half a step of the output
  lse          sum_j w_j e_j, sums, half a step of the value
A slot with a large e_j (a far one, whose bias is large) has no weight, so that the weighted sums are the ones that count."""
from __future__ import annotations

import numpy as np
import torch

from packed_testlib import HALF_STEP


class Mods:
    """The modifications of a call on the host."""

    def __init__(self, softcap=0.0, window=0, slopes=None, prefix=None, doc=None):
        self.softcap, self.window = softcap, window
        self.slopes = None if slopes is None else np.asarray(slopes, dtype=np.float32)
        self.prefix = None if prefix is None else np.asarray(prefix, dtype=np.int64)          # [n_seq]
        self.doc = None if doc is None else np.asarray(doc, dtype=np.int64)                   # [n_tokens]

    def device(self, B, dev):
        def t(x, dtype):
            return None if x is None else torch.tensor(x, dtype=dtype, device=dev)
        return B.Scores(self.softcap, self.window, t(self.slopes, torch.float32), t(self.prefix, torch.int32),
                        t(self.doc, torch.int32))

    def seen(self, s, first_row, base, n, length, causal=True):
        """[n, length] of sequence s: token t of it sees slot j."""
        p = base + np.arange(n)[:, None]
        j = np.arange(length)[None, :]
        ok = (j <= p) if causal else (j < base) & (p >= 0)
        if self.doc is not None:
            ok = ok & (j >= self.doc[first_row:first_row + n, None])
        if self.window:
            ok = ok & (p - j < self.window)
        if self.prefix is not None:
            ok = ok | (j < self.prefix[s])
        return ok


def attend64(q, k, v, ok, pos, mods, scale):
    """q [n, Hq, d], k, v [Hkv, L, d] (float64), ok [n, L], pos [n].  Returns O, lse and the first-order bounds
    (output's, lse's) of what is computed before the sums."""
    n, Hq, d = q.shape
    Hkv, L = k.shape[:2]
    G = Hq // Hkv
    O, A, eO = np.zeros_like(q), np.zeros_like(q), np.zeros_like(q)
    lse, eL = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    if L == 0:
        return O, lse, A, eO, eL
    dist = np.abs(pos[:, None] - np.arange(L)[None, :]).astype(np.float64)
    for hq in range(Hq):
        h = hq // G
        with np.errstate(all="ignore"):
            x = q[:, hq] @ k[h].T * scale
            e = (d + 2) * 2.0 ** -24 * (np.abs(q[:, hq]) @ np.abs(k[h]).T) * scale
            if mods.softcap:
                x = mods.softcap * np.tanh(x / mods.softcap)
                e = e + 2.0 ** -20 * np.abs(x)
            slope = 0.0 if mods.slopes is None else float(mods.slopes[hq])
            e = e + 4 * 2.0 ** -24 * (np.abs(x) + abs(slope) * (dist + 128))
            x = np.where(ok, x - slope * dist, -np.inf)
            m = x.max(axis=1, keepdims=True)
            w = np.exp(x - np.where(np.isneginf(m), 0.0, m))
            l = w.sum(axis=1, keepdims=True)
            w = np.where(ok, w / np.where(l == 0, 1.0, l), 0.0)
            rows = [np.flatnonzero(r) for r in ok] if not (np.isfinite(v[h]).all() and np.isfinite(e).all()) else None
            if rows is None:
                av = np.abs(v[h])
                O[:, hq], A[:, hq] = w @ v[h], w @ av
                eL[:, hq] = (w * e).sum(axis=1)
                eO[:, hq] = (w * e) @ av + A[:, hq] * eL[:, hq, None]
            else:                                      # hidden infinities and NaN: only the slots that a row sees
                for t, c in enumerate(rows):
                    vv = v[h][c]
                    O[t, hq], A[t, hq] = w[t, c] @ vv, w[t, c] @ np.abs(vv)
                    eL[t, hq] = (w[t, c] * e[t, c]).sum()
                    eO[t, hq] = (w[t, c] * e[t, c]) @ np.abs(vv) + A[t, hq] * eL[t, hq]
            lse[:, hq] = np.where(l[:, 0] == 0, -np.inf, (np.where(np.isneginf(m), 0.0, m) + np.log(l))[:, 0])
    return O, lse, A, eO, eL


def check(got_o, got_lse, ref, dtype, length, where=""):
    O, lse, A, eO, eL = ref
    sums = (length + 64) * 2.0 ** -24 + 2.0 ** -21
    p_round = HALF_STEP["bf16"] if dtype == "bf16" else 0.0
    assert np.array_equal(np.isnan(O), np.isnan(got_o)), f"{where}: NaN in other places"
    fine = np.isfinite(O)
    assert np.array_equal(O[~fine & ~np.isnan(O)], got_o[~fine & ~np.isnan(O)]), f"{where}: infinities differ"
    tol = (eO + (2 * sums + p_round) * A) * 1.01 + HALF_STEP[dtype] * 1.01 * np.abs(O) + 1e-37
    over = np.abs(got_o[fine] - O[fine]) - tol[fine]
    assert over.size == 0 or over.max() <= 0, f"{where}: output off by {np.abs(got_o[fine] - O[fine]).max():.3e} ({over.max():.3e} over its bound)"
    if got_lse is not None:
        assert np.array_equal(np.isneginf(lse), np.isneginf(got_lse)), f"{where}: empty rows differ"
        assert np.array_equal(np.isnan(lse), np.isnan(got_lse)), f"{where}: NaN lse in other places"
        ok = np.isfinite(lse)
        t2 = (eL[ok] + sums + 2.0 ** -23 * np.abs(lse[ok])) * 1.01
        off = np.abs(got_lse[ok] - lse[ok])
        assert (off <= t2).all(), f"{where}: lse off by {off.max():.3e}, {(off - t2).max():.3e} over its bound"
