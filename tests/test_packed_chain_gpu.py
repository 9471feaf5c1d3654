"""The compact cache goes on as pages: one handle for the library's own path and the packed calls."""
import numpy as np
import pytest
import torch

import samkv_testlib as T
from paper_2508_11661_b200 import binding as B
from paper_2508_11661_b200 import synth
from packed_testlib import attend64, check_rows, f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_compact_cache_moves_into_pages_and_both_attend_alike():
    w = synth.CONFIGS["cfg1"].replace(ctx_lens=(257, 64, 500), n_q_heads=8, n_kv_heads=2)
    inp = {n: t.to(DEV) for n, t in synth.make_inputs(w, "cpu").items()}
    run = T.DeviceRun(w, inp)
    S, d, page = run.S, w.head_dim, 32
    dtype = "bf16" if w.torch_dtype is torch.bfloat16 else "f32"
    off = torch.tensor([0, S], dtype=torch.int32, device=DEV)
    p = B.Packed(8, 2, d, off, S, dtype=dtype)
    own = B.samkv_workspace_bytes(run.shape, max(w.q_tokens, 1), run.capacity)
    run.handle = B.Handle.for_packed(p, at_least=own)
    assert run.handle.workspace.numel() == max(own, B.samkv_packed_workspace_bytes(p))
    run.sparsify()
    # the kept rows, [Hkv, capacity, d] as they are, into pages; nothing is rotated again
    n_pages = -(-S // page)
    Kp = torch.zeros((n_pages + 2, 2, page, d), dtype=w.torch_dtype, device=DEV)
    Vp = torch.zeros_like(Kp)
    table = torch.randperm(n_pages + 2)[:n_pages].to(torch.int32).view(1, -1).contiguous().to(DEV)
    pages = B.Pages(Kp, Vp, table)
    Kc, Vc = run.Kc[0, 0, :, :S], run.Vc[0, 0, :, :S]
    B.samkv_append(run.handle, p, Kc.permute(1, 0, 2), Vc.permute(1, 0, 2), pages)
    order = table[0].long()
    for pool, want in ((Kp, Kc), (Vp, Vc)):
        assert torch.equal(pool[order].permute(1, 0, 2, 3).reshape(2, -1, d)[:, :S], want)
    # queries over the pages, and over the compact cache, with the same handle in turn
    Q = inp["Qa"][0, 0]
    n = Q.shape[0]
    q = B.Packed(8, 2, d, torch.tensor([0, n], dtype=torch.int32, device=DEV), n, dtype=dtype)
    lens = torch.tensor([S], dtype=torch.int32, device=DEV)
    Kc64, Vc64 = f64(Kc), f64(Vc)
    ref = attend64(f64(Q), Kc64, Vc64, np.full(n, S), d ** -0.5)
    kept = run.Kc[0, 0].clone(), run.Vc[0, 0].clone()
    for _ in range(2):
        O, lse = torch.empty_like(Q), torch.empty((n, 8), dtype=torch.float32, device=DEV)
        B.samkv_paged_attn(run.handle, q, pages, lens, Q, 0.0, False, O, lse)
        check_rows(f64(O), f64(lse), ref, dtype, S)
        run.cache_len.fill_(S)
        Og, lse2 = run.attn(0, inp["Qa"][0], inp["Kq"][0], inp["Vq"][0])
        T.check_attention(w, kept[0], kept[1], S, Q, inp["Kq"][0, 0], inp["Vq"][0, 0], Og[0], lse2[0])
    assert run.poll() == 0
