"""Measured cases of the serving step around the paged cache: pages handed out on the GPU from request lengths, the
append with rotary positions of several axes, and attention whose scores are capped, biased by distance and masked.

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
    parts = [p.partition("*") for p in str(text).split(",")]
    return sum(([int(n)] * (int(times) if times else 1) for n, _, times in parts), [])


def _text(lens):
    return ",".join(str(int(n)) for n in lens)


def listed():
    """The head shapes are those of the package's benchmark configurations (4/2 heads of 64, 32/8 and 64/8 of 128)."""
    llama = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, dtype="bf16")
    wide = dict(n_q_heads=64, n_kv_heads=8, head_dim=128, dtype="bf16")
    tiny = dict(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype="f32")
    plain = dict(softcap=0.0, window=0, slopes=False, prefix=0, doc=0, tail=0)
    return [
        # ---- pages: finished requests give theirs back, the others get what their new tokens need ----
        # a decode step of 256 requests of mixed lengths, of which 16 have just finished
        dict(name="pages_decode", op="pages", new=_text([0 if i % 16 == 5 else 1 for i in range(256)]),
             cached=_text([(i * 977) % 8192 for i in range(256)]), done=16, pad=0, page=16, spare=300),
        # a step that takes up ten prompts of 2048 tokens next to ragged chunks and single tokens
        dict(name="pages_prompts", op="pages", new="2048*10,0,700,1*90,0,333,5000,1*60,0,17", cached="0*10,640,64,1000*90,0,63,4095,"
             "20480*60,1,129", done=41, pad=40, page=64, spare=1000),
        # ---- rotation by positions of several axes and append through the slot map ----
        # one decode step of 32 requests: text positions, the same on all three axes
        dict(name="axes_decode", op="axes", new="1*32", cached="1000*20,1,0,4095,63,64,65,127,128,2500,7,640,999", pad=0,
             page=64, interleaved=False, rot=128, axes=3, cycle=False, image=0, **llama),
        # ten prompts of 2048 tokens, each text around images of 24 x 24 patches (time, height, width)
        dict(name="axes_images", op="axes", new="2048*10", cached="0*10", pad=0, page=64, interleaved=False, rot=128, axes=3,
             cycle=False, image=24, **llama),
        # fp32, two axes taking turns over adjacent pairs, half of the head rotated, small pages, padding rows
        dict(name="axes_f32_ragged", op="axes", new="5,1,200,64,33", cached="11,0,500,16,47", pad=3, page=16, interleaved=True,
             rot=32, axes=2, cycle=True, image=7, **tiny),
        # ---- prompt attention with modified scores ----
        # the small fp32 configuration: one sequence of 4 documents of 256 tokens that do not see one another, and a question;
        # scores fall off with distance
        dict(name="prompt_f32_documents", op="prompt", new="1056", pad=0, **tiny, **{**plain, "slopes": True, "doc": 256, "tail": 32}),
        # ragged prompts of a model with distance slopes instead of rotation
        dict(name="prompt_ragged_slopes", op="prompt", new="1,64,2047,333,129,1,5000,18,777,1280", pad=30, **llama,
             **{**plain, "slopes": True}),
        # one layer of the 30 K token workload in one sequence: 20 documents of 1536 tokens behind a shared instruction of 64
        # that all see, a question of 128 that sees everything, scores capped
        dict(name="prompt_documents_cap", op="prompt", new="30912", pad=0, **llama,
             **{**plain, "softcap": 50.0, "prefix": 64, "doc": 1536, "tail": 128}),
        # ---- attention over the paged cache with modified scores ----
        # a decode step of 32 requests over 20480 cached tokens: scores capped, the last 4096 slots and 64 initial ones seen
        dict(name="decode_window_cap", op="paged", new="1*32", cached="20480*32", pad=0, page=64, causal=True, **llama,
             **{**plain, "softcap": 50.0, "window": 4096, "prefix": 64}),
        # one request over 100 K cached tokens with distance slopes: the work is split along the cache
        dict(name="decode_single_slopes", op="paged", new="1", cached="102400", pad=0, page=64, causal=True, **wide,
             **{**plain, "slopes": True}),
        # a chunk of 128 tokens over 100 K cached tokens, scores capped
        dict(name="chunk_cap", op="paged", new="128", cached="102400", pad=0, page=64, causal=True, **wide,
             **{**plain, "softcap": 30.0}),
        # a mixed fp32 batch: single tokens and chunks, empty and odd caches, small pages, all modifications
        dict(name="mixed_f32", op="paged", new="1,5,64,1,33,1", cached="700,0,131,15,2049,16", pad=2, page=16, causal=True, **tiny,
             **{**plain, "softcap": 20.0, "slopes": True, "prefix": 24, "doc": 100, "tail": 40, "window": 600}),
    ]


def _spread(rng, lo, hi):
    """An integer between lo and hi, evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["pages", "axes", "prompt", "prompt", "paged", "paged"])
    pad = rng.choice([0, 0, 1, 17, 100])
    if op == "pages":
        n_seq = _spread(rng, 1, 1500)
        most = 1 if rng.random() < 0.4 else max(1, min(5000, 40000 // n_seq))
        new = [rng.choice([0, 1, _spread(rng, 1, most)]) for _ in range(n_seq)]
        cached = [rng.choice([0, _spread(rng, 1, 20000)]) for _ in range(n_seq)]
        return dict(op=op, new=_text(new), cached=_text(cached), done=rng.choice([0, 2, 7, 30]), pad=pad,
                    page=rng.choice([16, 32, 64, 128, 256]), spare=_spread(rng, 1, 2000))
    heads = rng.choice([(4, 2, 64), (32, 8, 128), (64, 8, 128), (32, 8, 128), (6, 2, 64), (8, 8, 128), (5, 1, 128)])
    case = dict(op=op, n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=heads[2],
                dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), pad=pad)
    if op == "axes":
        n_seq = _spread(rng, 1, 64)
        new = [1] * n_seq if rng.random() < 0.4 else [_spread(rng, 1, 2000) for _ in range(min(n_seq, 10))]
        cached = [rng.choice([0, _spread(rng, 1, 4000)]) for _ in new]
        return dict(case, new=_text(new), cached=_text(cached), page=rng.choice([16, 32, 64, 128, 256]),
                    interleaved=rng.random() < 0.4, rot=rng.choice([heads[2], heads[2], heads[2] // 2, 16]),
                    axes=rng.choice([1, 2, 3, 3, 4]), cycle=rng.random() < 0.5, image=rng.choice([0, 1, 7, 16, 24, 33]))
    case.update(softcap=rng.choice([0.0, 20.0, 30.0, 50.0]), slopes=rng.random() < 0.3, prefix=rng.choice([0, 0, _spread(rng, 1, 600)]),
                window=rng.choice([0, 0, _spread(rng, 1, 6000)]), doc=rng.choice([0, 0, _spread(rng, 1, 2000)]),
                tail=rng.choice([0, 1, 32, 128]))
    if op == "prompt":
        left = 3e7 if case["dtype"] == "bf16" else 1.2e6           # pairs of one head: the largest listed case
        new = [_spread(rng, 1, 8192 if case["dtype"] == "bf16" else 1500) for _ in range(_spread(rng, 1, 50))]
        kept = [n for i, n in enumerate(new) if sum(m * m / 2 for m in new[:i + 1]) * heads[0] <= left * 32] or [1024]
        return dict(case, new=_text(kept))
    small = case["dtype"] == "f32"
    n_seq = _spread(rng, 1, 64)
    new = [1] * n_seq if rng.random() < 0.5 else [rng.choice([1, _spread(rng, 1, 64 if small else 500)]) for _ in range(min(n_seq, 10))]
    most = 4000 if small else max(200, min(100000, 600000 // len(new)))
    if max(new) > 1:
        most = max(64, min(most, 13000000 // sum(new)))            # pairs of one head: the chunk over 100 K tokens
    cached = [rng.choice([_spread(rng, 1, most), _spread(rng, 1, most), 0]) for _ in new]
    return dict(case, new=_text(new), cached=_text(cached), page=rng.choice([16, 32, 64, 128, 256]), causal=rng.random() < 0.85)


# ------------------------------------------------------------------------------------------------ inputs
def _offsets(lens):
    return torch.cumsum(torch.tensor([0] + lens), 0).to(torch.int32).to(DEV)


def _grid_positions(first, n, axes, image):
    """Positions [axes, n] of a prompt's tokens: 16 of text, an image of image x image patches, 16 of text, ...  Text moves on
    by one on every axis; an image stays where it starts on the first axis and counts rows and columns on the others."""
    out, at, pos = torch.empty((axes, n), dtype=torch.int64), 0, first
    while at < n:
        text = min(16 if image else n, n - at)
        out[:, at:at + text] = torch.arange(pos, pos + text)
        at, pos = at + text, pos + text
        patch = torch.arange(min(image * image, n - at))
        for a in range(axes):
            out[a, at:at + len(patch)] = pos + (0 if a == 0 else patch // image if a % 2 else patch % image) if image else 0
        at, pos = at + len(patch), pos + image
    return out


def _pair_axes(case):
    """The axis of every rotated pair: sections behind one another (the first half as long as the others), or in turns."""
    half, axes = case["rot"] // 2, case["axes"]
    if case["cycle"] or axes == 1:
        return [i % axes for i in range(half)]
    other = max(1, 2 * half // (2 * axes - 1))
    return [max(0, axes - 1 - (half - 1 - i) // other) for i in range(half)]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 6271 + 29)
    new = _lens(case["new"])
    T = sum(new) + case["pad"]
    st = dict(case=dict(case), n_tokens=T, new=new, offsets=_offsets(new))
    if case["op"] != "prompt":
        _cache_layout(case, st, g)
    if case["op"] == "pages":
        return st
    dt = DTYPES[case["dtype"]]
    Hq, Hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)

    # what the projections leave behind: rows of one fused matrix [T, Hq + 2 Hkv, d]
    fused = randn(T, Hq + 2 * Hkv, d)
    if case["op"] == "axes":
        fused = fused.to(dt)
        st["Q"], st["K"], st["V"] = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
        pos = [_grid_positions(c, n, case["axes"], case["image"]) for c, n in zip(st["cached"], new)]
        st["positions"] = torch.cat(pos + [torch.zeros((case["axes"], case["pad"]), dtype=torch.int64)], 1).to(torch.int32).to(DEV)
        st["Q_out"] = torch.zeros((T, Hq, d), dtype=dt, device=DEV)
        return st
    # capped scores are those of sharply peaked heads: a standard deviation of about 6
    gain = 6.0 if case["softcap"] else 1.0
    fused[:, :Hq] *= gain
    fused = fused.to(dt)
    st["Q"] = fused[:, :Hq]
    if case["op"] == "prompt":
        st["K"], st["V"] = fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    first = [0] * len(new) if case["op"] == "prompt" else st["cached"]
    st["softcap"], st["window"] = case["softcap"], case["window"]
    st["slopes"] = torch.exp2(-8.0 * (torch.arange(Hq, device=DEV) + 1) / Hq) if case["slopes"] else None
    st["prefix"] = torch.tensor([case["prefix"] + 3 * s for s in range(len(new))], dtype=torch.int32, device=DEV) if case["prefix"] else None
    st["doc_start"] = None
    if case["doc"]:
        # documents begin behind the prefix; the last `tail` tokens of a sequence see all of them
        start = torch.zeros(T, dtype=torch.int64)
        at = 0
        for c, n in zip(first, new):
            p = torch.arange(c, c + n) - case["prefix"]
            s = torch.where(p >= 0, torch.div(p, case["doc"], rounding_mode="floor") * case["doc"] + case["prefix"], 0)
            s[max(0, n - case["tail"]):] = 0
            start[at:at + n] = s
            at += n
        st["doc_start"] = start.to(torch.int32).to(DEV)
    st["O"] = torch.zeros((T, Hq, d), dtype=dt, device=DEV)
    st["lse"] = torch.zeros((T, Hq), dtype=torch.float32, device=DEV)
    return st


def _cache_layout(case, st, g):
    """Pools, block table and lengths; for the pages the state before the step, with the free ones on a stack."""
    new, cached, page = st["new"], _lens(case["cached"]), case["page"]
    n_seq = len(new)
    handed = case["op"] == "pages"
    held = [-(-c // page) for c in cached] if handed else [-(-(c + n) // page) for c, n in zip(cached, new)]
    done = [handed and case["done"] > 0 and s % case["done"] == case["done"] // 2 and new[s] == 0 for s in range(n_seq)]
    grown = sum(-(-(c + n) // page) for c, n in zip(cached, new)) if handed else sum(held)
    n_pages = grown + case.get("spare", 3)
    width = max(-(-(c + n) // page) for c, n in zip(cached, new)) + 2
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    seq = torch.repeat_interleave(torch.arange(n_seq), torch.tensor(held))
    col = torch.arange(len(seq)) - (torch.cumsum(torch.tensor(held), 0) - torch.tensor(held))[seq]
    table = torch.full((n_seq, width), -1, dtype=torch.int32, device=DEV)
    table[seq.to(DEV), col.to(DEV)] = order[:len(seq)]
    st.update(cached=cached, table=table, n_pages=n_pages, page=page)
    st["cache_len"] = torch.tensor([0 if f else c for c, f in zip(cached, done)], dtype=torch.int32, device=DEV)
    T = st["n_tokens"]
    if handed:
        st["lengths"] = torch.tensor(cached, dtype=torch.int32, device=DEV)
        st["done"] = torch.tensor(done, dtype=torch.bool, device=DEV)
        st["free"] = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
        st["free"][:n_pages - len(seq)] = order[len(seq):]
        st["n_free"] = torch.tensor([n_pages - len(seq)], dtype=torch.int32, device=DEV)
        st["n_back"], st["n_left"] = torch.zeros_like(st["n_free"]), torch.zeros_like(st["n_free"])
        for name, n in (("slots", T), ("positions", T), ("total_len", n_seq)):
            st[name] = torch.zeros(n, dtype=torch.int32, device=DEV)
        return
    Hkv, d, dt = case["n_kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
    st["Kp"] = torch.empty((n_pages, Hkv, page, d), dtype=dt, device=DEV)
    st["Vp"] = torch.empty_like(st["Kp"])
    for pool in (st["Kp"], st["Vp"]):
        for p0 in range(0, n_pages, 4096):
            p1 = min(p0 + 4096, n_pages)
            pool[p0:p1] = torch.randn((p1 - p0, Hkv, page, d), generator=g, device=DEV).to(dt)
    seq = torch.repeat_interleave(torch.arange(n_seq), torch.tensor(new)).to(DEV)
    pos = torch.arange(len(seq), device=DEV) - st["offsets"].long()[seq] + st["cache_len"].long()[seq]
    st["slots"] = torch.full((T,), -1, dtype=torch.int32, device=DEV)
    st["slots"][:len(seq)] = (table[seq, pos // page].long() * page + pos % page).to(torch.int32)


# ------------------------------------------------------------------------------------------------ plain forms
def _runs(lengths, total):
    """Of `total` things that belong to owners with so many each: whose each is, and which of its owner's."""
    who = torch.repeat_interleave(torch.arange(len(lengths), device=DEV), lengths, output_size=total)
    return who, torch.arange(total, device=DEV) - (torch.cumsum(lengths, 0) - lengths)[who]


def _plain_pages(st):
    page, table, free = st["page"], st["table"], st["free"]
    lengths, base, off = st["lengths"].long(), st["cache_len"].long(), st["offsets"].long()
    width, n_seq = table.shape[1], table.shape[0]
    # finished requests' pages go on top of the stack, the last one's last page first
    cols = torch.arange(width, device=DEV)
    back = st["done"][:, None] & (cols[None, :] < ((lengths + page - 1) // page)[:, None])
    rank = back.flatten().flip(0).cumsum(0).flip(0).reshape(n_seq, width)          # 1 for the last one
    where = torch.where(back, st["n_free"].long() + rank - 1, free.shape[0])
    grown = torch.cat([free, free[:1]])
    grown.scatter_(0, where.flatten(), table.flatten())
    free[:] = grown[:-1]
    st["n_back"][:] = st["n_free"] + back.sum().to(torch.int32)
    # the others' new pages come off it in order
    new = off[1:] - off[:-1]
    have = (base + page - 1) // page
    need = (base + new + page - 1) // page - have
    first = torch.cumsum(need, 0) - need
    k = cols[None, :] - have[:, None]
    fresh = (k >= 0) & (k < need[:, None])
    at = (st["n_back"].long() - 1 - first[:, None] - k).clamp(0, free.shape[0] - 1)
    table[:] = torch.where(fresh, free[at], table)
    st["n_left"][:] = st["n_back"] - need.sum().to(torch.int32)
    total = sum(st["new"])
    who, t = _runs(new, total)
    pos = base[who] + t
    st["slots"][:total] = (table[who, pos // page].long() * page + pos % page).to(torch.int32)
    st["positions"][:total] = pos.to(torch.int32)
    st["slots"][total:] = -1
    st["positions"][total:] = 0
    st["total_len"][:] = (base + new).to(torch.int32)
    return _pages_outputs(st)


def _pages_outputs(st):
    return dict(table=st["table"], slots=st["slots"], positions=st["positions"], total_len=st["total_len"], free=st["free"],
                n_back=st["n_back"], n_left=st["n_left"])


def _turned(x, angle, rot, interleaved):
    """x [T, H, d] in fp32 with its first `rot` elements rotated by the angles [T, rot / 2]."""
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _plain_axes(st):
    c = st["case"]
    rot, page, dt = c["rot"], c["page"], DTYPES[c["dtype"]]
    half = rot // 2
    freq = ROPE_BASE ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    axis = torch.tensor(_pair_axes(c), device=DEV)
    angle = st["positions"].double()[axis].T * freq
    live = st["slots"] >= 0
    total = sum(st["new"])                                  # (rows with a slot come first)
    q = _turned(st["Q"].float(), angle, rot, c["interleaved"]).to(dt)
    k = _turned(st["K"].float(), angle, rot, c["interleaved"]).to(dt)
    st["Q_out"][:] = torch.where(live[:, None, None], q, st["Q_out"])
    slot = st["slots"].long()[:total]
    st["Kp"][slot // page, :, slot % page] = k[:total]
    st["Vp"][slot // page, :, slot % page] = st["V"][:total]
    return dict(Q_out=st["Q_out"], Kp=st["Kp"], Vp=st["Vp"])


def _groups(st, first):
    """(sequences, tokens from, tokens to) whose scores fit 2 GB side by side, padded to the longest."""
    H, out, now = st["case"]["n_q_heads"], [], []
    for s, n in enumerate(st["new"]):
        both = now + [s]
        if now and len(both) * H * max(st["new"][i] for i in both) * max(first[i] + st["new"][i] for i in both) > 1 << 29:
            out, both = out + [now], [s]
        now = both
    parts = []
    for some in out + [now]:
        n, L = max(st["new"][i] for i in some), max(1, max(first[i] + st["new"][i] for i in some))
        step = max(1, (1 << 29) // (len(some) * H * L))
        parts += [(some, t, min(n, t + step)) for t in range(0, n, step)]
    return parts


def _plain_attention(st):
    c = st["case"]
    paged = c["op"] == "paged"
    first = st["cached"] if paged else [0] * len(st["new"])
    for some, t0, t1 in _groups(st, first):
        _attend_group(st, some, t0, t1, first, c, paged)
    return dict(O=st["O"], lse=st["lse"])


def _attend_group(st, some, t0, t1, first, c, paged):
    """Tokens t0 .. t1 of these sequences, side by side; sequences that are shorter leave rows unused."""
    Hq, Hkv, d = c["n_q_heads"], c["n_kv_heads"], c["head_dim"]
    causal = c.get("causal", True)
    idx = torch.tensor(some, device=DEV)
    base = torch.tensor([first[i] for i in some], device=DEV)[:, None]
    new = torch.tensor([st["new"][i] for i in some], device=DEV)[:, None]
    L = max(1, max(first[i] + st["new"][i] for i in some))
    t = torch.arange(t0, t1, device=DEV)[None, :]
    j = torch.arange(L, device=DEV)
    real = (t < new).expand(len(some), -1)
    rows = (st["offsets"].long()[idx][:, None] + t).clamp(max=st["n_tokens"] - 1)
    q = st["Q"][rows].float().reshape(len(some), t1 - t0, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4)
    if paged:
        page = c["page"]
        ids = st["table"][idx].long()[:, :-(-L // page)].clamp(min=0)
        k, v = (st[x][ids].transpose(1, 2).reshape(len(some), Hkv, -1, d)[:, :, :L].float() for x in ("Kp", "Vp"))
    else:
        at = (st["offsets"].long()[idx][:, None] + j).clamp(max=st["n_tokens"] - 1)
        k, v = (st[x][at].transpose(1, 2).float() for x in ("K", "V"))
    # which slots a token sees: [sequences, tokens, L]
    p = base + t
    end = p + 1 if causal else base.expand_as(p)
    low = torch.zeros_like(p) if st["doc_start"] is None else st["doc_start"].long()[rows]
    if st["window"]:
        low = torch.maximum(low, p - st["window"] + 1)
    seen = (j >= low[..., None]) & (j < end[..., None])
    if st["prefix"] is not None:
        seen |= j < torch.minimum(st["prefix"].long()[idx][:, None], base + new if causal else base)[..., None]
    x = torch.matmul(q, k[:, :, None].transpose(-1, -2)).mul_(1.0 / math.sqrt(d))      # [sequences, Hkv, G, tokens, L]
    if st["softcap"]:
        x = x.div_(st["softcap"]).tanh_().mul_(st["softcap"])
    if st["slopes"] is not None:
        x -= st["slopes"].reshape(1, Hkv, -1, 1, 1) * (p[..., None] - j).abs()[:, None, None].float()
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    w = x.sub_(m).exp_()
    l = w.sum(-1, keepdim=True)
    o = torch.matmul(w, v[:, :, None]) / torch.where(l > 0, l, 1.0)
    to = rows[real]
    st["O"][to] = o.permute(0, 3, 1, 2, 4).reshape(len(some), t1 - t0, Hq, d)[real].to(st["O"].dtype)
    st["lse"][to] = (m + l.log()).permute(0, 3, 1, 2, 4).reshape(len(some), t1 - t0, Hq)[real]


# ------------------------------------------------------------------------------------------------ one pass
def _plan(st):
    """What a user's program builds once and keeps: the descriptions of its tensors and a handle with its workspace."""
    from paper_2508_11661_b200 import binding as B
    c = st["case"]
    st["B"] = B
    shape = (1, 1, 64, "bf16") if c["op"] == "pages" else (c["n_q_heads"], c["n_kv_heads"], c["head_dim"], c["dtype"])
    st["packed"] = B.Packed(*shape[:3], st["offsets"], st["n_tokens"], max_seq_tokens=max(st["new"]), dtype=shape[3])
    st["handle"] = B.Handle.for_scores(st["packed"])
    if "Kp" in st:
        st["pages"] = B.Pages(st["Kp"], st["Vp"], st["table"])
    if c["op"] == "axes":
        st["rope"] = B.RopeAxes(c["rot"], _pair_axes(c), base=ROPE_BASE, interleaved=c["interleaved"])
    if c["op"] in ("prompt", "paged"):
        st["scores"] = B.Scores(softcap=st["softcap"], window=st["window"], slopes=st["slopes"], prefix_len=st["prefix"],
                                doc_start=st["doc_start"])


def run(st):
    op = st["case"]["op"]
    if not own:
        return _plain_pages(st) if op == "pages" else _plain_axes(st) if op == "axes" else _plain_attention(st)
    if "handle" not in st:
        _plan(st)
    B = st["B"]
    if op == "pages":
        B.samkv_release_pages(st["handle"], st["table"], st["page"], st["lengths"], st["done"], st["free"], st["n_free"], st["n_back"])
        B.samkv_page_tables(st["handle"], st["packed"], st["cache_len"], st["page"], st["table"], st["free"], st["n_back"],
                            st["n_left"], st["slots"], st["positions"], st["total_len"])
        return _pages_outputs(st)
    if op == "axes":
        B.samkv_append_axes(st["handle"], st["packed"], st["K"], st["V"], st["pages"], slots=st["slots"], rope=st["rope"],
                            positions=st["positions"], Q=st["Q"], Q_out=st["Q_out"])
        return dict(Q_out=st["Q_out"], Kp=st["Kp"], Vp=st["Vp"])
    if op == "prompt":
        B.samkv_prefill_scores(st["handle"], st["packed"], st["Q"], st["K"], st["V"], 0.0, st["scores"], st["O"], st["lse"])
    else:
        B.samkv_paged_attn_scores(st["handle"], st["packed"], st["pages"], st["cache_len"], st["Q"], 0.0, st["case"]["causal"],
                                  st["scores"], st["O"], st["lse"])
    return dict(O=st["O"], lse=st["lse"])


# ------------------------------------------------------------------------------------------------ floors
def _visible(case, first, n):
    """Of one sequence: (pairs, slots that any token sees), from the masks' ends."""
    causal = case.get("causal", True)
    L = first + n if causal else first
    pre = min(case["prefix"], L)
    p = torch.arange(first, first + n)
    low = torch.zeros_like(p)
    if case["doc"]:
        behind = p - case["prefix"]
        low = torch.where(behind >= 0, torch.div(behind, case["doc"], rounding_mode="floor") * case["doc"] + case["prefix"], 0)
        low[max(0, n - case["tail"]):] = 0
    if case["window"]:
        low = torch.maximum(low, p - case["window"] + 1)
    end = p + 1 if causal else torch.full_like(p, first)
    low = torch.maximum(low, torch.tensor(pre))
    pairs = int((end - low).clamp(min=0).sum()) + n * pre
    some = (end > low)
    return pairs, pre + (int(end[some].max() - low[some].min()) if bool(some.any()) else 0)


def work(case):
    """Bytes: every input that counts read once, results written once.  Attention: the slots that some token of a sequence
    sees; operations: two per product and sum of the two matrix products over the visible (query, key) pairs."""
    new = _lens(case["new"])
    total = sum(new)
    if case["op"] == "pages":
        page, cached = case["page"], _lens(case["cached"])
        grown = sum(-(-(c + n) // page) - -(-c // page) for c, n in zip(cached, new))
        back = sum(-(-c // page) for s, c in enumerate(cached) if case["done"] and s % case["done"] == case["done"] // 2 and new[s] == 0)
        return {"bytes": 4 * (2 * (grown + back) + 2 * (total + case["pad"]) + 4 * len(new)), "flops": 4 * total}
    e = 2 if case["dtype"] == "bf16" else 4
    Hq, Hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    if case["op"] == "axes":
        return {"bytes": 2 * total * (Hq + 2 * Hkv) * d * e + 4 * total * (1 + case["axes"]), "flops": 3 * total * (Hq + Hkv) * case["rot"]}
    first = [0] * len(new) if case["op"] == "prompt" else _lens(case["cached"])
    pairs, rows = (sum(x) for x in zip(*(_visible(case, c, n) for c, n in zip(first, new) if n)))
    return {"bytes": 2 * total * Hq * d * e + 2 * rows * Hkv * d * e + 4 * total * Hq, "flops": 4 * pairs * Hq * d}


# ------------------------------------------------------------------------------------------------ definition, 64 bits
def exact(case, seed):
    """Each operator from its definition: a page, a token or the rows of one head at a time."""
    st = prepare(case, seed)
    if case["op"] == "pages":
        return _exact_pages(st)
    if case["op"] == "axes":
        return _exact_axes(st, case)
    d64 = torch.float64
    Hq, Hkv, d, T = case["n_q_heads"], case["n_kv_heads"], case["head_dim"], st["n_tokens"]
    G = Hq // Hkv
    O = torch.zeros((T, Hq, d), dtype=d64, device=DEV)
    lse = torch.zeros((T, Hq), dtype=d64, device=DEV)
    causal = case.get("causal", True)
    at = 0
    for s, n in enumerate(st["new"]):
        c = 0 if case["op"] == "prompt" else st["cached"][s]
        L = c + n if causal else c
        pre = 0 if st["prefix"] is None else min(int(st["prefix"][s]), L)
        if case["op"] == "prompt":
            keys, values = st["K"][at:at + n], st["V"][at:at + n]
        else:
            slots = torch.arange(L, device=DEV)
            ids = st["table"][s].long()[torch.div(slots, case["page"], rounding_mode="floor")]
            keys, values = (st[x][ids, :, slots % case["page"]] for x in ("Kp", "Vp"))
        step = max(1, (1 << 26) // max(1, G * L))
        for t0 in range(0, n, step):
            p = torch.arange(c + t0, c + min(n, t0 + step), device=DEV)
            rows = slice(at + t0, at + t0 + len(p))
            low = torch.zeros_like(p) if st["doc_start"] is None else st["doc_start"][rows].long()
            # (only the slots that some row can see take part)
            j = torch.arange(L, device=DEV)
            ok = (j[None, :] <= p[:, None]) if causal else torch.ones((len(p), L), dtype=torch.bool, device=DEV)
            ok = ok & (j[None, :] >= low[:, None])
            if case["window"]:
                ok = ok & (p[:, None] - j[None, :] < case["window"])
            ok = ok | (j < pre)[None, :]
            cols = torch.nonzero(ok.any(0)).flatten()
            ok = ok[:, cols]
            far = (p[:, None] - cols[None, :]).abs().to(d64)
            for h in range(Hkv):
                heads = slice(h * G, (h + 1) * G)
                x = torch.einsum("tgd,ld->gtl", st["Q"][rows, heads].to(d64), keys[cols, h].to(d64)) / math.sqrt(d)
                if case["softcap"]:
                    x = case["softcap"] * torch.tanh(x / case["softcap"])
                if case["slopes"]:
                    x = x - st["slopes"][heads].to(d64)[:, None, None] * far
                x = torch.where(ok, x, torch.full_like(x, -math.inf))
                norm = torch.logsumexp(x, -1) if len(cols) else torch.full(x.shape[:2], -math.inf, dtype=d64, device=DEV)
                w = torch.where(ok, torch.exp(x - torch.where(norm.isinf(), torch.zeros_like(norm), norm)[..., None]), torch.zeros_like(x))
                O[rows, heads] = torch.einsum("gtl,ld->tgd", w, values[cols, h].to(d64))
                lse[rows, heads] = norm.T
        at += n
    return dict(O=O, lse=lse)


def _exact_pages(st):
    page, table = st["page"], st["table"].tolist()
    n, free = int(st["n_free"]), st["free"].tolist()
    done, lengths, base = st["done"].tolist(), st["lengths"].tolist(), st["cache_len"].tolist()
    stack = free[:n]
    for s in reversed(range(len(table))):
        if done[s]:
            stack += [table[s][c] for c in reversed(range(-(-lengths[s] // page)))]
    free[:len(stack)] = stack
    back = len(stack)
    slots, positions = [-1] * st["n_tokens"], [0] * st["n_tokens"]
    at = 0
    for s, new in enumerate(st["new"]):
        for t in range(new):
            pos = base[s] + t
            if pos % page == 0:
                table[s][pos // page] = stack.pop()
            slots[at], positions[at] = table[s][pos // page] * page + pos % page, pos
            at += 1

    def i32(x):
        return torch.tensor(x, dtype=torch.int32, device=DEV)
    return dict(table=i32(table), slots=i32(slots), positions=i32(positions), total_len=i32([b + m for b, m in zip(base, st["new"])]),
                free=i32(free), n_back=i32([back]), n_left=i32([len(stack)]))


def _exact_axes(st, case):
    d64, half, rot, T = torch.float64, case["rot"] // 2, case["rot"], st["n_tokens"]
    Q, Kp, Vp = st["Q_out"].to(d64), st["Kp"].to(d64), st["Vp"].to(d64)
    one = slice(0, rot, 2) if case["interleaved"] else slice(0, half)
    two = slice(1, rot, 2) if case["interleaved"] else slice(half, rot)
    axis = _pair_axes(case)
    slots = st["slots"].long()
    for t0 in range(0, T, 1024):
        rows = torch.arange(t0, min(T, t0 + 1024), device=DEV)
        rows = rows[slots[rows] >= 0]
        turn = torch.empty((len(rows), 1, half), dtype=torch.complex128, device=DEV)
        for i in range(half):
            angle = st["positions"][axis[i]][rows].to(d64) * ROPE_BASE ** (-i / half)
            turn[:, 0, i] = torch.polar(torch.ones_like(angle), angle)
        for src in ("Q", "K"):
            x = st[src][rows].to(d64)
            z = torch.complex(x[..., one].contiguous(), x[..., two].contiguous()) * turn
            x[..., one], x[..., two] = z.real, z.imag
            if src == "Q":
                Q[rows] = x
        page, row = torch.div(slots[rows], case["page"], rounding_mode="floor"), slots[rows] % case["page"]
        Kp[page, :, row] = x
        Vp[page, :, row] = st["V"][rows].to(d64)
    return dict(Q_out=Q, Kp=Kp, Vp=Vp)
