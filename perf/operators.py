"""Measured cases of the packed and paged operators: prompt attention of documents packed behind one another, the
rotating append to a paged cache, and attention of new tokens over a paged cache.

`run` with `own = False` computes each operator from elementary torch operations; with `own = True` it makes the calls
a user makes of this package.  Sequence lengths are written as text, "1536*20,7" meaning twenty of 1536 and one of 7.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ROPE_BASE = 500000.0


# ------------------------------------------------------------------------------------------------ cases
def _lens(text):
    out = []
    for part in str(text).split(","):
        n, _, times = part.partition("*")
        out += [int(n)] * (int(times) if times else 1)
    return out


def _text(lens):
    return ",".join(str(int(n)) for n in lens)


def listed():
    """The head shapes are those of the package's benchmark configurations (4/2 heads of 64, 32/8 and 64/8 of 128)."""
    llama = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, dtype="bf16")
    wide = dict(n_q_heads=64, n_kv_heads=8, head_dim=128, dtype="bf16")
    tiny = dict(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype="f32")
    return [
        # ---- prompt attention: documents are prefilled independently of one another, packed into one call ----
        # a single user query without documents: the time is launch and latency
        dict(name="prefill_query", op="prefill", new="17", pad=0, sharp=False, **llama),
        # the small fp32 configuration that parity work runs on: 4 documents of 256 tokens
        dict(name="prefill_f32_documents", op="prefill", new="256*4", pad=0, sharp=False, **tiny),
        # a retriever's documents as they come: one token, odd lengths, long ones, padding rows behind the last
        dict(name="prefill_ragged", op="prefill", new="1,64,2047,333,129,1,5000,18,777,1280", pad=30, sharp=True, **llama),
        # 20 documents of 1536 tokens: one layer of one request of the 30 K token workload
        dict(name="prefill_documents", op="prefill", new="1536*20", pad=0, sharp=True, **llama),
        # 50 documents of 2048 tokens, 64 query heads: one layer of the 100 K token workload
        dict(name="prefill_stress", op="prefill", new="2048*50", pad=0, sharp=False, **wide),
        # ---- rotation and append: the step between the projections and attention ----
        # one decode step of 32 requests
        dict(name="append_decode", op="append", new="1*32", cached="1000*20,1,0,4095,63,64,65,127,128,2500,7,640,999",
             pad=0, page=64, interleaved=False, rot=128, far=0, **llama),
        # one layer of a prompt of 20480 tokens in 10 requests, at positions far into a long conversation
        dict(name="append_prompt", op="append", new="2048*10", cached="0*10", pad=0, page=64, interleaved=False, rot=128,
             far=1000000, **llama),
        # fp32, adjacent pairs, half of the head rotated, small pages
        dict(name="append_f32_ragged", op="append", new="5,1,200,64,33", cached="11,0,500,16,47", pad=3, page=16,
             interleaved=True, rot=32, far=0, **tiny),
        # ---- attention over the paged cache ----
        # one decode step of 32 requests over 20480 cached tokens each
        dict(name="decode_batch", op="paged_attn", new="1*32", cached="20480*32", pad=0, page=64, causal=True, **llama),
        # one decode step of a single request over 100 K cached tokens: the work is split along the cache
        dict(name="decode_single", op="paged_attn", new="1", cached="102400", pad=0, page=64, causal=True, **wide),
        # a query chunk of 128 tokens over 100 K cached tokens
        dict(name="chunk_stress", op="paged_attn", new="128", cached="102400", pad=0, page=64, causal=True, **wide),
        # a mixed fp32 batch: single tokens and chunks, empty and odd caches, small pages
        dict(name="mixed_f32", op="paged_attn", new="1,5,64,1,33,1", cached="700,0,131,15,2049,16", pad=2, page=16,
             causal=True, **tiny),
    ]


def _spread(rng, lo, hi):
    """An integer between lo and hi, evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prefill", "append", "paged_attn"])
    heads = rng.choice([(4, 2, 64), (32, 8, 128), (64, 8, 128), (32, 8, 128), (6, 2, 64), (8, 8, 128), (5, 1, 128)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    case = dict(op=op, n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=heads[2], dtype=dtype,
                pad=rng.choice([0, 0, 1, 17, 100]))
    small = dtype == "f32"
    if op == "prefill":
        n_seq = _spread(rng, 1, 50)
        most = 1024 if small else 8192
        new = [_spread(rng, 1, most) for _ in range(n_seq)]
        case.update(new=_text(new), sharp=rng.random() < 0.5)
        return case
    n_seq = _spread(rng, 1, 64)
    case["page"] = rng.choice([16, 32, 64, 128, 256])
    if op == "append":
        new = [1] * n_seq if rng.random() < 0.4 else [_spread(rng, 1, 2000) for _ in range(min(n_seq, 10))]
        cached = [rng.choice([0, _spread(rng, 1, 4000)]) for _ in new]
        case.update(new=_text(new), cached=_text(cached), interleaved=rng.random() < 0.4,
                    rot=rng.choice([heads[2], heads[2], heads[2] // 2, 16]), far=rng.choice([0, 0, 5000, 1000000]))
        return case
    if rng.random() < 0.5:
        new = [1] * n_seq
    else:
        n_seq = min(n_seq, 12)
        new = [rng.choice([1, _spread(rng, 1, 64 if small else 600)]) for _ in range(n_seq)]
    most = 4000 if small else max(200, min(100000, 600000 // n_seq))
    cached = [rng.choice([_spread(rng, 1, most), _spread(rng, 1, most), 0]) for _ in new]
    case.update(new=_text(new), cached=_text(cached), causal=rng.random() < 0.85)
    return case


# ------------------------------------------------------------------------------------------------ inputs
def _rotation(positions, rot, base, interleaved, x):
    """Rotates the first `rot` elements of x [T, H, d] by the angles of `positions` [T]; angles in 64 bits."""
    half = rot // 2
    freq = base ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half)
    angle = positions.to(torch.float64)[:, None] * freq[None, :]
    cos, sin = angle.cos()[:, None, :].to(x.dtype), angle.sin()[:, None, :].to(x.dtype)
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _page_layout(case):
    new, cached, page = _lens(case["new"]), _lens(case["cached"]), case["page"]
    need = [-(-(c + n) // page) for c, n in zip(cached, new)]
    return need, max(max(need), 1) + 1, sum(need) + 3


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 13)
    dt = DTYPES[case["dtype"]]
    Hq, Hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    new = _lens(case["new"])
    T = sum(new) + case["pad"]
    st = dict(case=dict(case), n_tokens=T, new=new)
    off = [0]
    for n in new:
        off.append(off[-1] + n)
    st["offsets"] = torch.tensor(off, dtype=torch.int32, device=DEV)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)

    if case["op"] == "prefill":
        # what the projections leave behind: rows of one fused matrix [T, Hq + 2 Hkv, d], queries and keys rotated
        # with every document starting at position 0
        fused = torch.empty((T, Hq + 2 * Hkv, d), dtype=dt, device=DEV)
        pos = torch.cat([torch.arange(n, device=DEV) for n in new] + [torch.zeros(case["pad"], device=DEV)])
        q, k = randn(T, Hq, d), randn(T, Hkv, d)
        if case["sharp"]:                       # a few strong channels and a sink at each document's first token
            k[..., :: d // 4] *= 4.0
            k[st["offsets"][:-1].long().clamp(max=T - 1)] *= 2.0
        fused[:, :Hq] = _rotation(pos, d, ROPE_BASE, False, q).to(dt)
        fused[:, Hq:Hq + Hkv] = _rotation(pos, d, ROPE_BASE, False, k).to(dt)
        fused[:, Hq + Hkv:] = randn(T, Hkv, d).to(dt)
        st["Q"], st["K"], st["V"] = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    else:
        need, width, n_pages = _page_layout(case)
        page = case["page"]
        cached = _lens(case["cached"])
        order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        table = torch.full((len(new), width), -1, dtype=torch.int32, device=DEV)
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = order[at:at + n]
            at += n
        st["table"] = table
        st["cached"] = cached
        st["cache_len"] = torch.tensor(cached, dtype=torch.int32, device=DEV)
        st["Kp"] = torch.empty((n_pages, Hkv, page, d), dtype=dt, device=DEV)
        st["Vp"] = torch.empty_like(st["Kp"])
        for pool in (st["Kp"], st["Vp"]):
            for p0 in range(0, n_pages, 4096):
                p1 = min(p0 + 4096, n_pages)
                pool[p0:p1] = randn(p1 - p0, Hkv, page, d).to(dt)
        if case["op"] == "append":
            fused = randn(T, Hq + 2 * Hkv, d).to(dt)
            st["Q"], st["K"], st["V"] = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
            pos = [torch.arange(case["far"] + c, case["far"] + c + n) for c, n in zip(cached, new)]
            st["positions"] = torch.cat(pos + [torch.zeros(case["pad"], dtype=torch.int64)]).to(torch.int32).to(DEV)
            st["Q_out"] = torch.zeros((T, Hq, d), dtype=dt, device=DEV)
        else:
            st["Q"] = randn(T, Hq, d).to(dt)
    if case["op"] != "append":
        st["O"] = torch.zeros((T, Hq, d), dtype=dt, device=DEV)
        st["lse"] = torch.zeros((T, Hq), dtype=torch.float32, device=DEV)
    if own:
        _plan(st)
    return st


def _plan(st):
    """What a user's program builds once and keeps: the descriptions of its tensors and a handle with its workspace."""
    from paper_2508_11661_b200 import binding as B
    c = st["case"]
    st["B"] = B
    st["packed"] = B.Packed(c["n_q_heads"], c["n_kv_heads"], c["head_dim"], st["offsets"], st["n_tokens"],
                            max_seq_tokens=max(st["new"]), dtype=c["dtype"])
    if c["op"] != "prefill":
        st["pages"] = B.Pages(st["Kp"], st["Vp"], st["table"])
    if c["op"] == "append":
        st["rope"] = B.Rope(c["rot"], base=ROPE_BASE, interleaved=c["interleaved"])
    st["handle"] = B.Handle.for_packed(st["packed"])


# ------------------------------------------------------------------------------------------------ one pass
def _attend(q, k, v, first, causal, scale):
    """q [n, Hq, d], k and v [Hkv, L, d] in fp32.  Query t sees the first `first + t + 1` keys, or the first `first`
    without the causal tail.  Returns o [n, Hq, d] and the log of the softmax denominators [n, Hq]."""
    n, Hq, d = q.shape
    Hkv, L = k.shape[0], k.shape[1]
    G = Hq // Hkv
    o = torch.zeros_like(q)
    lse = torch.full((n, Hq), -math.inf, device=q.device, dtype=q.dtype)
    step = max(1, (1 << 28) // max(1, Hq * L))
    for t0 in range(0, n, step):
        t1 = min(n, t0 + step)
        rows = q[t0:t1].reshape(t1 - t0, Hkv, G, d).permute(1, 0, 2, 3).reshape(Hkv, (t1 - t0) * G, d)
        seen = torch.arange(t0, t1, device=q.device).repeat_interleave(G) + first + 1 if causal else \
            torch.full(((t1 - t0) * G,), first, device=q.device)
        last = max(1, first + t1 if causal else first)
        s = torch.matmul(rows, k[:, :last].transpose(1, 2)) * scale
        hidden = torch.arange(last, device=q.device)[None, :] >= seen[:, None]
        s.masked_fill_(hidden, -math.inf)
        m = s.max(dim=-1, keepdim=True).values
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        p = s.sub_(m).exp_()
        l = p.sum(dim=-1, keepdim=True)
        out = torch.matmul(p, v[:, :last]) / torch.where(l > 0, l, torch.ones_like(l))
        o[t0:t1] = out.reshape(Hkv, t1 - t0, G, d).permute(1, 0, 2, 3).reshape(t1 - t0, Hq, d)
        lse[t0:t1] = (m + l.log()).reshape(Hkv, t1 - t0, G).permute(1, 0, 2).reshape(t1 - t0, Hq)
    return o, lse


def _from_pages(pool, table_row, length):
    """The first `length` rows of a sequence: [Hkv, length, d] in fp32."""
    Hkv, page, d = pool.shape[1:]
    n = -(-length // page)
    return pool[table_row[:n].long()].permute(1, 0, 2, 3).reshape(Hkv, n * page, d)[:, :length].float()


def _plain(st):
    c = st["case"]
    scale = 1.0 / math.sqrt(c["head_dim"])
    at = 0
    if c["op"] == "append":
        page = c["page"]
        dt = DTYPES[c["dtype"]]
        pos, total = st["positions"], sum(st["new"])
        q = _rotation(pos, c["rot"], ROPE_BASE, c["interleaved"], st["Q"].float()).to(dt)
        k = _rotation(pos, c["rot"], ROPE_BASE, c["interleaved"], st["K"].float()).to(dt)
        st["Q_out"][:total] = q[:total]
        seq = torch.repeat_interleave(torch.arange(len(st["new"]), device=DEV),
                                      torch.tensor(st["new"], device=DEV), output_size=total)
        slot = torch.arange(total, device=DEV) - st["offsets"].long()[seq] + st["cache_len"].long()[seq]
        where = st["table"].long()[seq, slot // page]
        st["Kp"][where, :, slot % page] = k[:total]
        st["Vp"][where, :, slot % page] = st["V"][:total]
        return dict(Q_out=st["Q_out"], Kp=st["Kp"], Vp=st["Vp"])
    for s, n in enumerate(st["new"]):
        rows = slice(at, at + n)
        at += n
        if c["op"] == "prefill":
            o, lse = _attend(st["Q"][rows].float(), st["K"][rows].permute(1, 0, 2).float(),
                             st["V"][rows].permute(1, 0, 2).float(), 0, True, scale)
        else:
            first = st["cached"][s]
            length = max(1, first + n if c["causal"] else first)
            o, lse = _attend(st["Q"][rows].float(), _from_pages(st["Kp"], st["table"][s], length),
                             _from_pages(st["Vp"], st["table"][s], length), first, c["causal"], scale)
        st["O"][rows] = o.to(st["O"].dtype)
        st["lse"][rows] = lse
    return dict(O=st["O"], lse=st["lse"])


def run(st):
    if not own:
        return _plain(st)
    if "handle" not in st:
        _plan(st)
    B, c = st["B"], st["case"]
    if c["op"] == "prefill":
        B.samkv_prefill(st["handle"], st["packed"], st["Q"], st["K"], st["V"], 0.0, st["O"], st["lse"])
        return dict(O=st["O"], lse=st["lse"])
    if c["op"] == "append":
        B.samkv_append(st["handle"], st["packed"], st["K"], st["V"], st["pages"], st["cache_len"], st["rope"],
                       positions=st["positions"], Q=st["Q"], Q_out=st["Q_out"])
        return dict(Q_out=st["Q_out"], Kp=st["Kp"], Vp=st["Vp"])
    B.samkv_paged_attn(st["handle"], st["packed"], st["pages"], st["cache_len"], st["Q"], 0.0, c["causal"], st["O"],
                       st["lse"])
    return dict(O=st["O"], lse=st["lse"])


# ------------------------------------------------------------------------------------------------ floors
def work(case):
    """Bytes: queries, keys and values read once, results written once.  Operations: two per product and sum of the
    two matrix products over the visible (query, key) pairs."""
    e = 2 if case["dtype"] == "bf16" else 4
    Hq, Hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    new = _lens(case["new"])
    total = sum(new)
    if case["op"] == "append":
        moved = 2 * total * (Hq + 2 * Hkv) * d * e
        return {"bytes": moved + 4 * total, "flops": 3 * total * (Hq + Hkv) * case["rot"]}
    cached = [0] * len(new) if case["op"] == "prefill" else _lens(case["cached"])
    causal = case["op"] == "prefill" or case["causal"]
    pairs = sum(n * c + (n * (n + 1) // 2 if causal else 0) for n, c in zip(new, cached))
    kv_rows = sum(c + (n if causal else 0) for n, c in zip(new, cached) if n > 0)
    return {"bytes": 2 * total * Hq * d * e + 2 * kv_rows * Hkv * d * e + 4 * total * Hq,
            "flops": 4 * pairs * Hq * d}


# ------------------------------------------------------------------------------------------------ definition, 64 bits
def exact(case, seed):
    """Each operator from its definition in 64 bits: one query row of one head at a time in the formulas, many rows at
    a time in the arithmetic."""
    st = prepare(case, seed)
    d64 = torch.float64
    Hq, Hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    G = Hq // Hkv
    T = st["n_tokens"]
    if case["op"] == "append":
        half = case["rot"] // 2
        Q, Kp, Vp = torch.zeros((T, Hq, d), dtype=d64, device=DEV), st["Kp"].to(d64), st["Vp"].to(d64)
        t = 0
        for s, n in enumerate(st["new"]):
            for t0 in range(0, n, 1024):
                m = min(1024, n - t0)
                angle = torch.empty((m, half), dtype=d64, device=DEV)
                for i in range(half):
                    first = case["far"] + st["cached"][s] + t0
                    angle[:, i] = torch.arange(first, first + m, dtype=d64, device=DEV) * ROPE_BASE ** (-i / half)
                turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]
                for src, dst in (("Q", "q"), ("K", "k")):
                    x = st[src][t + t0:t + t0 + m].to(d64)
                    y = x.clone()
                    one = slice(0, case["rot"], 2) if case["interleaved"] else slice(0, half)
                    two = slice(1, case["rot"], 2) if case["interleaved"] else slice(half, case["rot"])
                    z = torch.complex(x[..., one].contiguous(), x[..., two].contiguous()) * turn
                    y[..., one], y[..., two] = z.real, z.imag
                    if dst == "q":
                        Q[t + t0:t + t0 + m] = y
                    else:
                        k = y
                v = st["V"][t + t0:t + t0 + m].to(d64)
                slots = torch.arange(t0, t0 + m, device=DEV) + st["cached"][s]
                page = st["table"][s].long()[torch.div(slots, case["page"], rounding_mode="floor")]
                Kp[page, :, slots % case["page"]] = k
                Vp[page, :, slots % case["page"]] = v
            t += n
        return dict(Q_out=Q, Kp=Kp, Vp=Vp)
    O = torch.zeros((T, Hq, d), dtype=d64, device=DEV)
    lse = torch.zeros((T, Hq), dtype=d64, device=DEV)
    t = 0
    for s, n in enumerate(st["new"]):
        for h in range(Hkv):
            if case["op"] == "prefill":
                first, tail = 0, True
                k, v = st["K"][t:t + n, h].to(d64), st["V"][t:t + n, h].to(d64)
            else:
                first, tail = st["cached"][s], case["causal"]
                L = first + n if tail else first
                ids = st["table"][s, :-(-L // case["page"])].long()
                k = st["Kp"][ids, h].reshape(-1, d)[:L].to(d64)
                v = st["Vp"][ids, h].reshape(-1, d)[:L].to(d64)
            step = max(1, (1 << 26) // max(1, G * k.shape[0]))
            for t0 in range(0, n, step):
                m = min(step, n - t0)
                seen = [first + t0 + i + 1 if tail else first for i in range(m)]
                L = seen[-1]
                rows = slice(t + t0, t + t0 + m)
                heads = slice(h * G, (h + 1) * G)
                if L == 0:
                    lse[rows, heads] = -math.inf
                    continue
                x = torch.einsum("tgd,ld->tgl", st["Q"][rows, heads].to(d64), k[:L]) / math.sqrt(d)
                limit = torch.tensor(seen, device=DEV)[:, None, None]
                x = torch.where(torch.arange(L, device=DEV)[None, None, :] < limit, x, torch.full_like(x, -math.inf))
                norm = torch.logsumexp(x, dim=-1)
                O[rows, heads] = torch.einsum("tgl,ld->tgd", torch.exp(x - norm[..., None]), v[:L])
                lse[rows, heads] = norm
        t += n
    return dict(O=O, lse=lse)
