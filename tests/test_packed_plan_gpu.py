"""How calls with many sequences are laid out: up to 32 sequences, one warp's share (512) and more, in every kernel."""
import numpy as np
import pytest
import torch

from packed_testlib import PagedCase, attend64, check_rows, f64
from test_packed_gpu import check_paged, check_prefill, randn, run_paged, run_prefill

pytestmark = pytest.mark.gpu
COUNTS = [31, 32, 33, 200, 512, 513, 1500]


def lengths(n_seq, most, seed, empty=0.3):
    """Ragged lengths, a share of them zero, single tokens among them."""
    r = np.random.default_rng(seed)
    x = r.integers(1, most + 1, n_seq)
    x[r.random(n_seq) < empty] = 0
    x[r.random(n_seq) < 0.2] = 1
    x[0], x[-1] = 0, 1                                   # an empty first sequence and a short last one
    return [int(v) for v in x]


def on_the_host(c):
    """The 64-bit form reads the pools once per sequence."""
    c.Kp, c.Vp = c.Kp.cpu().double(), c.Vp.cpu().double()
    return c


@pytest.mark.parametrize("n_seq", COUNTS)
@pytest.mark.parametrize("dtype,new,hint,Hq,Hkv", [("bf16", 2, 2, 8, 2), ("bf16", 12, 0, 8, 2), ("f32", 2, 2, 8, 2),
                                                   ("f32", 18, 0, 16, 1)])
def test_sequences_over_pages(n_seq, dtype, new, hint, Hq, Hkv):
    """bf16 decode and tensor-memory kernels, fp32 with 8 rows and (16 heads of one KV head, from 200 sequences on) 64."""
    r = np.random.default_rng(n_seq)
    c = PagedCase(lengths(n_seq, new, n_seq), [int(x) for x in r.integers(0, 90, n_seq)], Hq, Hkv, 64, 16, dtype, seed=300, pad=2)
    O, lse = run_paged(c, max_seq=hint)
    check_paged(on_the_host(c), O, lse)


@pytest.mark.parametrize("n_seq", COUNTS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts(n_seq, dtype):
    lens = lengths(n_seq, 70 if n_seq < 100 else 12, n_seq + 1)
    T = sum(lens) + 3
    q, k, v = (randn(T, h, 64, dtype=dtype, seed=301 + i) for i, h in enumerate((4, 2, 2)))
    O, lse = run_prefill(q, k, v, lens, dtype)
    check_prefill(q, k, v, lens, dtype, O, lse)


@pytest.mark.parametrize("n_seq", [2, 33, 512, 513, 700])
def test_one_long_chunk_among_many_sequences_runs_in_waves(n_seq):
    """A captured step has room for many sequences of which few are active: one chunk over keys that L2 cannot hold, some
    single tokens, the others empty.  Repeated, with the results of every call compared bit for bit."""
    long = n_seq // 2
    new, cached = [0] * n_seq, [0] * n_seq
    for s in range(0, n_seq, max(1, n_seq // 12)):
        new[s], cached[s] = 1, 50 + s
    new[long], cached[long] = 300, 70001
    c = PagedCase(new, cached, 8, 2, 128, 64, "bf16", seed=305)
    O, lse = run_paged(c)
    for _ in range(5):
        O2, lse2 = run_paged(c)
        assert torch.equal(O, O2) and torch.equal(lse, lse2)
    q, o, l = f64(c.Q), f64(O), f64(lse)
    on_the_host(c)
    for s in range(n_seq):
        if new[s] == 0:
            continue
        at, n = int(c.starts[s]), new[s]
        rows = np.array(sorted({0, n // 2, n - 1, min(31, n - 1), min(32, n - 1)}))
        k, v = c.slots(c.Kp, s, cached[s] + n), c.slots(c.Vp, s, cached[s] + n)
        ref = attend64(q[at + rows], k, v, cached[s] + rows + 1, 128 ** -0.5)
        check_rows(o[at + rows], l[at + rows], ref, "bf16", cached[s] + n, f"sequence {s}")
