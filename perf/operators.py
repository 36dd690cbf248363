"""The paged-cache operators: their plain forms, the framework's calls, and the cases that are timed.

Two kinds of case.  "append" puts new tokens' keys and values into a paged cache, the keys (and the
queries of the same tokens) rotated by their positions on the way; with a 4-bit cache it also reads the
cached rows back as values.  "attend" is attention of new tokens' queries over such a cache, causal
among the new tokens, with an optional sliding window.  A cache holds bf16, fp32, or 4-bit codes with
one (scale, lowest value) pair per 32 channels of a token.

Page layouts (one layer, in front of everything here):
  bf16, fp32   [pages][2 (K, V)][kv_heads][page_size][head_dim]
  4 bits       [pages][kv_heads][page_size / 16 blocks], a block of 16 tokens being
               K codes   32-bit words [token][t 0..3][group j], channels 32 j + 8 t + 0..7, low nibble first
               V codes   32-bit words [token pair][g 0..7][group j]: the low half holds the even token's
                         channels 32 j + 4 g + 0..3, the high half the odd token's
               K scale   bf16 [token pair][group][token of the pair]
               K lowest  bf16 [token][group]
               V scale   as K scale
               V lowest  as K scale
  value = lowest + scale * code
"""
import math

import torch

own = False

LLAMA = {"q_heads": 32, "kv_heads": 8, "head_dim": 128}
QWEN = {"q_heads": 28, "kv_heads": 4, "head_dim": 128}
TINY = {"q_heads": 4, "kv_heads": 1, "head_dim": 64}


def listed():
    return [
        # one decode step of a batch: every sequence stores one token (latency)
        {"name": "append_decode_b16", "op": "append", "cache": "bf16", **LLAMA, "batch": 16, "page": 16,
         "len_lo": 513, "len_hi": 4097, "new_lo": 1, "new_hi": 1, "rot": 128, "interleaved": False},
        # the prompts of a batch, whole and ragged
        {"name": "append_prompts_b16", "op": "append", "cache": "bf16", **LLAMA, "batch": 16, "page": 64,
         "len_lo": 512, "len_hi": 4096, "new_lo": 512, "new_hi": 4096, "rot": 128, "interleaved": False},
        # a small fp32 model whose rotation turns half of the channels, neighbours paired; short odd pieces
        {"name": "append_f32_pieces", "op": "append", "cache": "f32", **TINY, "batch": 5, "page": 16,
         "len_lo": 300, "len_hi": 600, "new_lo": 1, "new_hi": 300, "rot": 32, "interleaved": True},
        # prompts stored in 4 bits and handed on as values (what a context's prompt pool is loaded from)
        {"name": "append4_prompts_b16", "op": "append", "cache": "int4", **LLAMA, "batch": 16, "page": 64,
         "len_lo": 512, "len_hi": 4096, "new_lo": 512, "new_hi": 4096, "rot": 128, "interleaved": False},
        # one sequence decoding (latency)
        {"name": "attend_b1", "op": "attend", "cache": "bf16", **LLAMA, "batch": 1, "page": 16,
         "len_lo": 1025, "len_hi": 1025, "new_lo": 1, "new_hi": 1, "window": 0, "lse": False},
        # the ordinary decode batch: ragged, prompts and what was generated since
        {"name": "attend_b16", "op": "attend", "cache": "bf16", **LLAMA, "batch": 16, "page": 64,
         "len_lo": 1537, "len_hi": 5121, "new_lo": 1, "new_hi": 1, "window": 0, "lse": False},
        # a large batch with long contexts and seven query heads per KV head
        {"name": "attend_qwen_b64", "op": "attend", "cache": "bf16", **QWEN, "batch": 64, "page": 32,
         "len_lo": 2048, "len_hi": 16384, "new_lo": 1, "new_hi": 1, "window": 0, "lse": True},
        # pieces of long prompts worked through together, over what is cached already
        {"name": "attend_pieces_b4", "op": "attend", "cache": "bf16", **LLAMA, "batch": 4, "page": 64,
         "len_lo": 1400, "len_hi": 5200, "new_lo": 700, "new_hi": 1300, "window": 0, "lse": False},
        # a small fp32 model with a sliding window
        {"name": "attend_f32_window", "op": "attend", "cache": "f32", **TINY, "batch": 7, "page": 16,
         "len_lo": 1, "len_hi": 2000, "new_lo": 1, "new_hi": 1, "window": 777, "lse": True},
        # one sequence decoding over a long context in 4 bits (latency)
        {"name": "attend4_b1", "op": "attend", "cache": "int4", **LLAMA, "batch": 1, "page": 16,
         "len_lo": 4099, "len_hi": 4099, "new_lo": 1, "new_hi": 1, "window": 0, "lse": False},
        # a decode batch over long contexts in 4 bits
        {"name": "attend4_b16", "op": "attend", "cache": "int4", **LLAMA, "batch": 16, "page": 64,
         "len_lo": 4096, "len_hi": 32768, "new_lo": 1, "new_hi": 1, "window": 0, "lse": False},
        # pieces of long prompts over a context in 4 bits
        {"name": "attend4_pieces_b2", "op": "attend", "cache": "int4", **LLAMA, "batch": 2, "page": 64,
         "len_lo": 5000, "len_hi": 9000, "new_lo": 600, "new_hi": 1000, "window": 0, "lse": False},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    cache = rng.choice(["bf16", "bf16", "int4", "int4", "f32"])
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = {"kv_heads": kv, "q_heads": kv * rng.choice([1, 2, 4, 5, 7, 8]), "head_dim": rng.choice([64, 128, 128])}
    c = {"op": rng.choice(["append", "attend", "attend"]), "cache": cache, **heads, "page": rng.choice([16, 32, 64, 128])}
    if c["op"] == "append":
        c["batch"] = _log(rng, 1, 64)
        c["new_lo"] = 1
        c["new_hi"] = rng.choice([1, 1, _log(rng, 2, max(2, min(2048, 16000 // c["batch"])))])
        c["len_lo"] = c["new_hi"] + rng.randint(0, 100)
        c["len_hi"] = c["len_lo"] + _log(rng, 1, 1000)
        c["rot"] = rng.choice([0, c["head_dim"] // 4, c["head_dim"], c["head_dim"]])
        c["interleaved"] = rng.random() < 0.3
        return c
    kind = rng.choice(["one", "one", "few", "many"])
    c["lse"] = rng.random() < 0.5
    if kind == "many":      # pieces of prompts
        c["batch"] = rng.randint(1, 4)
        most = min(300 if cache == "f32" else 1000, 16000 // c["q_heads"])
        c["new_lo"] = _log(rng, 17, most)
        c["new_hi"] = c["new_lo"] + rng.randint(0, 100)
        c["len_lo"] = c["new_hi"] + rng.randint(0, 500)
        c["len_hi"] = c["len_lo"] + _log(rng, 1, 1000 if cache == "f32" else 4000)
    else:
        c["batch"] = _log(rng, 1, 64)
        c["new_lo"] = 1
        c["new_hi"] = 1 if kind == "one" else rng.randint(2, 9)     # 2 to 9: checking drafted tokens
        c["len_lo"] = c["new_hi"] + rng.randint(0, 63)
        c["len_hi"] = c["len_lo"] + _log(rng, 1, min(16000, 300000 // c["batch"]) // (4 if cache == "f32" else 1))
    c["window"] = rng.choice([0, 0, 0, _log(rng, 1, 5000)])
    return c


def _bf16(x):
    return x.to(torch.float32).to(torch.bfloat16)


def _quantise(x):
    """fp64 [..., d] -> codes [..., d / 32, 32] (fp64), scale and lowest value [..., d / 32] (bf16)."""
    x = x.unflatten(-1, (-1, 32))
    low, high = x.amin(-1), x.amax(-1)
    fine = torch.isfinite(x).all(-1)
    lowest = _bf16(torch.where(fine, low, 0.0))
    scale = _bf16(torch.where(fine, high / 15 - low / 15, math.nan))
    s = scale.double()[..., None]
    codes = torch.where(s > 0, ((x - lowest.double()[..., None]) / s).round().clamp(0, 15), 0.0)
    return codes, scale, lowest


def _values(codes, scale, lowest):
    return (lowest.float()[..., None] + scale.float()[..., None] * codes.float()).flatten(-2)


def _pack(K, V, page):
    """K, V fp64 [pages, kv_heads, page, d] -> the 4-bit pages, uint8 [pages, kv_heads, bytes]."""
    n, h, _, d = K.shape
    g = d // 32
    kc, ks, kl = _quantise(K)
    vc, vs, vl = _quantise(V)
    nib = torch.arange(8, device=K.device) * 4
    kw = kc.long().reshape(n, h, page // 16, 16, g, 4, 8).transpose(-3, -2)                 # token, t, group, 8
    kw = (kw << nib).sum(-1).to(torch.int32)
    vw = vc.long().reshape(n, h, page // 16, 8, 2, g, 8, 4).permute(0, 1, 2, 3, 6, 5, 4, 7)  # pair, g, group, token, 4
    vw = (vw.flatten(-2) << nib).sum(-1).to(torch.int32)
    pairs = lambda a: a.reshape(n, h, page // 16, 8, 2, g).transpose(-1, -2).contiguous()  # noqa: E731
    raw = [kw, vw, pairs(ks), kl.reshape(n, h, page // 16, 16, g), pairs(vs), pairs(vl)]
    raw = [a.contiguous().reshape(n, h, page // 16, -1).view(torch.uint8) for a in raw]
    return torch.cat(raw, -1).reshape(n, h, -1)


def _unpack(raw, d):
    """Blocks uint8 [..., bytes of a block] -> K and V values, fp32 [..., 16, d]."""
    g = d // 32
    kw, vw, ks, kl, vs, vl = raw.split([8 * d, 8 * d, 32 * g, 32 * g, 32 * g, 32 * g], -1)
    nib = torch.arange(8, device=raw.device, dtype=torch.int32) * 4
    lead = raw.shape[:-1]
    kc = (kw.contiguous().view(torch.int32).reshape(*lead, 16, 4, g, 1) >> nib) & 15
    kc = kc.transpose(-3, -2).reshape(*lead, 16, g, 32)
    vc = (vw.contiguous().view(torch.int32).reshape(*lead, 8, 8, g, 1) >> nib) & 15
    vc = vc.unflatten(-1, (2, 4)).movedim(-2, -4).transpose(-3, -2).reshape(*lead, 16, g, 32)
    pairs = lambda a: a.contiguous().view(torch.bfloat16).reshape(*lead, 8, g, 2).transpose(-1, -2).reshape(*lead, 16, g)  # noqa: E731
    kl = kl.contiguous().view(torch.bfloat16).reshape(*lead, 16, g)
    return _values(kc, pairs(ks), kl), _values(vc, pairs(vs), pairs(vl))


def _lengths(c):
    """Tokens in the cache after the step, and new tokens, per sequence: part of the case, not of the seed."""
    gen = torch.Generator().manual_seed(c["batch"] * 7919 + c["len_hi"] * 31 + c["new_hi"])
    r = lambda lo, hi: torch.randint(lo, hi + 1, (c["batch"],), generator=gen)  # noqa: E731
    lens, new = r(c["len_lo"], c["len_hi"]), r(c["new_lo"], c["new_hi"])
    if c["op"] == "append" and c["new_lo"] == c["len_lo"]:
        new = lens.clone()      # whole prompts into an empty cache
    return lens, torch.minimum(new, lens)


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    B, hq, hk, d, page = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    io = torch.float32 if c["cache"] == "f32" else torch.bfloat16
    lens, new = _lengths(c)
    per = -(-int(lens.max()) // page)
    need = -(-lens // page)
    n_pages = int(need.sum()) + 3
    # pages in a mixed order, as a pool gives them out; table entries that no token needs are -1
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((B, per), -1, dtype=torch.int32)
    used = torch.arange(per)[None, :] < need[:, None]
    table[used] = order[: int(need.sum())]
    starts = torch.zeros(B + 1, dtype=torch.int32)
    starts[1:] = new.cumsum(0)
    T = int(starts[-1])
    rand = lambda *shape: torch.randn(*shape, generator=gen, device=dev)  # noqa: E731
    st = {"case": c, "lens": lens.to(torch.int32).to(dev), "table": table.to(dev), "starts": starts.to(dev),
          "T": T, "max_new": int(new.max()), "max_len": int(lens.max()),
          # sequence of every new token, and its place in the cache
          "seq": torch.repeat_interleave(torch.arange(B), new).to(dev)}
    st["pos"] = (torch.cat([torch.arange(int(a), int(b)) for a, b in zip(lens - new, lens)])).to(dev)
    st["single"] = T == B and c["new_hi"] == 1
    if c["op"] == "append":
        # one buffer as a projection leaves it: q, k and v of a token side by side
        qkv = rand(T, hq + 2 * hk, d).to(io)
        st["q"], st["k"], st["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        st["q_out"] = torch.zeros(T, hq, d, dtype=io, device=dev)
        if c["rot"]:
            st["inv_freq"] = (500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])).float().to(dev)
        if c["cache"] == "int4":
            st["pages"] = torch.zeros(1, n_pages, hk, page // 16 * (16 * d + 128 * (d // 32)), dtype=torch.uint8, device=dev)
            st["K"] = torch.zeros(B, hk, st["max_new"], d, dtype=io, device=dev)
            st["V"] = torch.zeros_like(st["K"])
            st["first"] = (lens - new).to(torch.int32).to(dev)
        else:
            st["pages"] = torch.zeros(1, n_pages, 2, hk, page, d, dtype=io, device=dev)
    else:
        st["q"] = (rand(T, hq, d) * 2 * math.sqrt(d)).to(io)
        st["out"] = torch.zeros(T, hq, d, dtype=io, device=dev)
        st["lse"] = torch.zeros(T, hq, device=dev) if c["lse"] else None
        # keys scaled so that the logits have a deviation of 2; a few channels carry an offset, as keys do
        off = torch.zeros(d, device=dev)
        off[5::29] = 2 / math.sqrt(d)
        if c["cache"] == "int4":
            k = ((rand(n_pages, hk, page, d) / math.sqrt(d)) + off).to(io).double()
            v = (rand(n_pages, hk, page, d) / math.sqrt(d)).to(io).double()
            st["pages"] = _pack(k, v, page)[None]
            del k, v
        else:
            st["pages"] = (rand(n_pages, 2, hk, page, d) / math.sqrt(d)).to(io)
            st["pages"][:, 0] += off.to(io)
            st["pages"] = st["pages"][None]
    if own:
        import paper_2605_29873_b200 as mkv
        kinds = {"bf16": mkv.MKV_BF16, "f32": mkv.MKV_F32, "int4": mkv.MKV_INT4}
        st["ctx"] = mkv.PagedKV(st["pages"], hq, hk, d, page, B, kv_dtype=kinds[c["cache"]],
                                io_dtype=mkv.MKV_F32 if io == torch.float32 else mkv.MKV_BF16)
        if c["op"] == "append" and c["rot"]:
            st["ctx"].set_rotation(st["inv_freq"], interleaved=c["interleaved"])
    return st


def run(state):
    if own:
        return _run_own(state)
    return _append(state) if state["case"]["op"] == "append" else _attend(state)


def _run_own(st):
    c, ctx = st["case"], st["ctx"]
    starts = None if st["single"] else st["starts"]
    if c["op"] == "append":
        ctx.append(0, st["q"], st["k"], st["v"], st["lens"], st["table"], q_out=st["q_out"], starts=starts)
        if c["cache"] != "int4":
            return st["q_out"], st["pages"]
        ctx.read(0, st["lens"], st["table"], st["K"], st["V"], first=st["first"])
        return st["q_out"], st["K"], st["V"]
    ctx.attend(0, st["q"], st["lens"], st["table"], st["out"], starts=starts, max_new=st["max_new"],
               window=c["window"], lse=st["lse"])
    return (st["out"], st["lse"]) if c["lse"] else (st["out"],)


def _rotate(x, st, wide):
    """x [T, heads, d] turned by its tokens' positions, in fp64 where `wide`, else in fp32."""
    c = st["case"]
    x = x.to(torch.float64 if wide else torch.float32)
    r = c["rot"]
    if r == 0:
        return x
    angle = st["pos"].double()[:, None] * st["inv_freq"].double()
    cos, sin = angle.cos().to(x.dtype)[:, None], angle.sin().to(x.dtype)[:, None]
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., : r // 2], x[..., r // 2: r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _append(st):
    c = st["case"]
    page = c["page"]
    st["q_out"].copy_(_rotate(st["q"], st, False))
    if c["cache"] == "int4":
        row = st["pos"] - st["first"].long()[st["seq"]]
        # codes are next to borders: 64 bits up to the code
        st["K"][st["seq"], :, row] = _values(*_quantise(_rotate(st["k"], st, True))).to(st["K"].dtype)
        st["V"][st["seq"], :, row] = _values(*_quantise(st["v"].double())).to(st["V"].dtype)
        return st["q_out"], st["K"], st["V"]
    at = st["table"][st["seq"], st["pos"] // page].long()
    st["pages"][0][at, 0, :, st["pos"] % page] = _rotate(st["k"], st, False).to(st["k"].dtype)
    st["pages"][0][at, 1, :, st["pos"] % page] = st["v"]
    return st["q_out"], st["pages"]


def _attend(st):
    c = st["case"]
    B, hq, hk, d, page, n = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page"], st["max_new"]
    at = st["table"].long().clamp_min(0)
    if c["cache"] == "int4":
        raw = st["pages"][0][at]                                       # [B, pages, kv_heads, bytes]
        K, V = _unpack(raw.unflatten(-1, (page // 16, -1)), d)           # [B, pages, kv_heads, blocks, 16, d]
        K, V = (x.flatten(3, 4).transpose(1, 2).flatten(2, 3) for x in (K, V))
    else:
        kv = st["pages"][0][at].float()                                # [B, pages, 2, kv_heads, page, d]
        K, V = (kv[:, :, i].transpose(1, 2).flatten(2, 3) for i in (0, 1))
    q = torch.zeros(B, n, hq, d, device=K.device)
    row = torch.arange(st["T"], device=K.device) - st["starts"].long()[st["seq"]]
    q[st["seq"], row] = st["q"].float()
    q = q.reshape(B, n, hk, hq // hk, d).transpose(1, 2).flatten(2, 3)   # [B, kv_heads, n * group, d]
    s = q @ K.transpose(-1, -2) / math.sqrt(d)
    j = torch.arange(K.shape[2], device=K.device)
    new = (st["starts"][1:] - st["starts"][:-1]).long()
    p = (st["lens"].long() - new)[:, None] + torch.arange(n, device=K.device)   # positions of the queries
    seen = (j <= p[..., None]) & (j < st["lens"].long()[:, None, None])
    if c["window"]:
        seen &= j > p[..., None] - c["window"]
    s = s.unflatten(2, (n, -1)).masked_fill_(~seen[:, None, :, None], -math.inf).flatten(2, 3)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    s = s.sub_(m).exp_()
    total = s.sum(-1, keepdim=True)
    o = (s @ V) / torch.where(total == 0, 1.0, total)
    o = o.unflatten(2, (n, -1)).transpose(1, 2).flatten(2, 3)            # [B, n, q_heads, d]
    st["out"].copy_(o[st["seq"], row])
    if not c["lse"]:
        return (st["out"],)
    lse = (m + total.log()).squeeze(-1).unflatten(2, (n, -1)).transpose(1, 2).flatten(2, 3)
    st["lse"].copy_(lse[st["seq"], row])
    return st["out"], st["lse"]


def _seen(c):
    """Rows of the cache that the new tokens see: per sequence, the rows that must be read, and over all tokens."""
    lens, new = _lengths(c)
    w = c["window"] or 1 << 30
    rows = torch.minimum(lens, new + (w - 1))
    total = 0
    for L, m in zip(lens.tolist(), new.tolist()):
        p = torch.arange(L - m, L)
        total += int(torch.minimum(p + 1, torch.tensor(w)).sum())
    return rows, total


def work(case):
    c = case
    d, hq, hk = c["head_dim"], c["q_heads"], c["kv_heads"]
    size = 4 if c["cache"] == "f32" else 2
    row = 2 * d * size if c["cache"] != "int4" else d + 8 * (d // 32)     # K and V of one token of a head, cached
    lens, new = _lengths(c)
    T = int(new.sum())
    if c["op"] == "append":
        # q, k, v read; rotated q and the cache written; in 4 bits the values handed on as well
        moved = T * (2 * hq + 2 * hk) * d * size + T * hk * row
        if c["cache"] == "int4":
            moved += T * hk * 2 * d * size
        return {"bytes": moved, "flops": T * (hq + hk) * c["rot"] * 3}
    rows, total = _seen(c)
    moved = int(rows.sum()) * hk * row + 2 * T * hq * d * size + (4 * T * hq if c["lse"] else 0)
    return {"bytes": moved, "flops": 4 * total * hq * d}


def exact(case, seed):
    """The same from the definition in 64 bits, sequence by sequence."""
    st = prepare(case, seed)
    c = st["case"]
    B, hq, hk, d, page = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    lens, starts, table = st["lens"].tolist(), st["starts"].tolist(), st["table"].tolist()
    if c["op"] == "append":
        def turned(x, pos):
            y = x.clone()
            for i in range(c["rot"] // 2):
                a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + c["rot"] // 2)
                w = pos * float(st["inv_freq"][i])
                y[..., a] = x[..., a] * w.cos() - x[..., b] * w.sin()
                y[..., b] = x[..., a] * w.sin() + x[..., b] * w.cos()
            return y

        def coded(x):
            y = torch.empty_like(x)
            for g in range(0, d, 32):
                z = x[..., g:g + 32]
                low = z.min(-1, keepdim=True).values
                step = (z.max(-1, keepdim=True).values - low).div(15).float().bfloat16().double()
                low = low.float().bfloat16().double()
                n = torch.clamp(torch.round((z - low) / torch.where(step == 0, 1.0, step)), 0, 15)
                y[..., g:g + 32] = low + torch.where(step == 0, 0.0, n * step)
            return y

        pos = st["pos"].double()[:, None]
        q, k, v = turned(st["q"].double(), pos), turned(st["k"].double(), pos), st["v"].double()
        if c["cache"] == "int4":
            K, V = st["K"].double(), st["V"].double()
            for b in range(B):
                n = starts[b + 1] - starts[b]
                K[b, :, :n] = coded(k[starts[b]:starts[b + 1]]).transpose(0, 1)
                V[b, :, :n] = coded(v[starts[b]:starts[b + 1]]).transpose(0, 1)
            return q, K, V
        pages = st["pages"].double()
        for b in range(B):
            n = starts[b + 1] - starts[b]
            p = torch.arange(lens[b] - n, lens[b], device=q.device)
            at = torch.tensor(table[b], device=q.device)[p // page]
            pages[0, at, 0, :, p % page] = k[starts[b]:starts[b + 1]]
            pages[0, at, 1, :, p % page] = v[starts[b]:starts[b + 1]]
        return q, pages
    out = torch.zeros(st["T"], hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((st["T"], hq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, L = starts[b + 1] - starts[b], lens[b]
        if n == 0 or L == 0:
            continue
        at = torch.tensor(table[b][: -(-L // page)], device="cuda")
        one = st["pages"][0, at]
        if c["cache"] == "int4":
            # from the bytes, a nibble at a time
            raw = one.reshape(at.numel(), hk, page // 16, -1).long()
            g = d // 32
            t, ch = torch.arange(16, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
            j, r = ch // 32, ch % 32
            kb = t * (d // 2) + ((r // 8) * g + j) * 4 + r % 8 // 2
            vb = 8 * d + (t // 2) * d + ((r // 4) * g + j) * 4 + t % 2 * 2 + r % 4 // 2
            sb = ((t // 2) * g + j) * 4 + t % 2 * 2
            lb = (t * g + j) * 2
            base = 16 * d
            num = lambda o: ((raw[..., o] + 256 * raw[..., o + 1]) << 16).int().view(torch.float32).double()  # noqa: E731
            nib = lambda o: (raw[..., o] >> (4 * (r % 2))) & 15  # noqa: E731
            K = num(base + 32 * g + lb) + num(base + sb) * nib(kb)
            V = num(base + 96 * g + sb) + num(base + 64 * g + sb) * nib(vb)
            K, V = (x.transpose(0, 1).reshape(hk, -1, d)[:, :L] for x in (K, V))
        else:
            K, V = (one[:, i].transpose(0, 1).reshape(hk, -1, d)[:, :L].double() for i in (0, 1))
        at_q = torch.arange(L - n, L, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")[None]
        hide = j > at_q
        if c["window"]:
            hide |= j <= at_q - c["window"]
        for h in range(hq):
            s = st["q"][starts[b]:starts[b + 1], h].double() @ K[h * hk // hq].T * d ** -0.5
            s[hide] = -math.inf
            lse[starts[b]:starts[b + 1], h] = torch.logsumexp(s, -1)
            out[starts[b]:starts[b + 1], h] = torch.softmax(s, -1) @ V[h * hk // hq]
    return (out, lse) if c["lse"] else (out,)
