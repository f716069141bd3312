"""Rotary positions, appends to a paged cache and attention over an 8-bit cache: measured cases and their plain forms.

What surrounds a decode step of a serving engine: queries and keys get their rotary positions (one axis for text, several for images
and video), new keys and values go into the paged cache (16-bit, or 8-bit with one scale per block and KV head), and attention reads
the 8-bit cache (a token per request, over all pages or a page table from the selector; a few drafted tokens; a chunk of a prompt).
Head counts, page sizes, budgets and context lengths are those of this repository's configurations and benchmark; the chat, draft,
chunk and video cases use generic ones.

A case is a dict of plain values:
  kind        "rope" | "append" (16- or 32-bit cache) | "qappend" (8-bit cache) | "attend" (8-bit cache)
  batch       requests
  lo, hi      tokens that the requests' sequences hold, the new ones included, spread over lo .. hi
  nlo, nhi    new tokens per request (rotated, appended or asking), spread over nlo .. nhi; "rope": batch * nhi tokens in one row
  pad         rows behind the last request's tokens that belong to nobody
  hq, hkv     query heads, KV heads
  page        tokens per page
  dtype       element type of queries, keys and values ("bf16" | "f32")
  fmt         "attend": codes of the cache, "int8" | "e4m3" ("qappend": "e4m3", whose codes are numbers that can be compared)
  layout      cache [block, head, token, dim] "HND" | [block, token, head, dim] "NHD"
  axes        axes of a position, 1 (text) .. 4
  rot         dimensions that are rotated
  inter       pairs of neighbouring dimensions are rotated, not halves
  fused       query, key and value rows are slices of one projection's rows
  budget      "attend": tokens in each KV head's page table; 0: all pages
"""
import math

import torch

own = False
D = 128
BASE = 500000.0   # of the rotary frequencies
CODE_MAX = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -100   # a page whose largest magnitude is below this is stored as zeros
FIRST = {1: [64], 2: [32, 64], 3: [16, 40, 64], 4: [16, 32, 48, 64]}   # of 64 frequencies, the ends of the axes' sections


def _case(name, kind, batch, lo, hi, nlo=1, nhi=1, pad=0, hq=32, hkv=8, page=16, dtype="bf16", fmt="e4m3", layout="HND", axes=1,
          rot=128, inter=False, fused=False, budget=0):
    c = dict(kind=kind, batch=batch, lo=lo, hi=hi, nlo=nlo, nhi=nhi, pad=pad, hq=hq, hkv=hkv, page=page, dtype=dtype, fmt=fmt,
             layout=layout, axes=axes, rot=rot, inter=inter, fused=fused, budget=budget)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # 24 chat requests, a token each, at (time, height, width) positions: the smallest call
        _case("rope_decode_24_thw", "rope", 24, 0, 0, axes=3),
        # a video prompt of 8K patches, rows sliced out of the fused projection
        _case("rope_video_8k_thw", "rope", 1, 0, 0, 8191, 8191, axes=3, fused=True),
        # a decode step's new token of 32 requests, an odd one of them padding, into a 16-bit cache
        _case("append_decode_32", "append", 32, 15700, 16384, pad=1),
        # chunks of five prompts, 4K tokens together, into a cache whose tokens lie together
        _case("append_chunks_5", "append", 5, 1100, 9001, 301, 1500, layout="NHD", fused=True),
        # the benchmark's headline batch, a token each, into the 8-bit cache
        _case("qappend_decode_8x32k", "qappend", 8, 31900, 32768),
        # twelve prompts of ragged lengths, prefilled together
        _case("qappend_prompts_12", "qappend", 12, 211, 2048, 211, 2048, pad=7, fused=True),
        # the benchmark's headline batch kept dense: all of an 8-bit cache, a token per request
        _case("attend_8x32k_int8", "attend", 8, 31900, 32768, fmt="int8"),
        # the same batch over the selector's page tables
        _case("attend_8x32k_listed", "attend", 8, 31900, 32768, fmt="int8", budget=2048),
        # one long document, 16 query heads per KV head
        _case("attend_1x1m_g16", "attend", 1, 1048500, 1048500, hkv=2),
        # chat traffic, ragged and short, 32-token pages
        _case("attend_chat_24", "attend", 24, 211, 9001, page=32, layout="NHD"),
        # drafted tokens of six requests, verified in one pass
        _case("attend_drafts_6", "attend", 6, 3001, 12000, 2, 5, pad=3, fmt="int8"),
        # a chunk of a long prompt
        _case("attend_chunk_1k", "attend", 1, 16301, 16301, 1024, 1024),
    ]


def draw(rng):
    def spread(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    kind = rng.choices(["rope", "append", "qappend", "attend"], [2, 2, 2, 6])[0]
    hq, hkv = rng.choices([(32, 8), (32, 4), (32, 2), (28, 4), (40, 8)], [5, 1, 1, 1, 1])[0]
    page = rng.choices([16, 32, 64], [4, 1, 1])[0]
    layout = rng.choice(["HND", "NHD"])
    dtype = rng.choice(["bf16", "bf16", "f32"]) if kind in ("rope", "append") else "bf16"
    axes, inter, fused = rng.choice([1, 1, 2, 3, 4]), rng.random() < 0.3, rng.random() < 0.5
    rot = rng.choice([128, 128, 96, 64])
    more = dict(hq=hq, hkv=hkv, page=page, dtype=dtype, layout=layout, axes=axes, rot=rot, inter=inter, fused=fused)
    if kind == "rope":
        batch = spread(1, 64)
        n = spread(1, 8191 // batch)
        return _case("", kind, batch, 0, 0, n, n, rng.choice([0, 3]), **more)
    if kind != "attend":
        batch = spread(1, 64)
        nhi = 1 if rng.random() < 0.4 else spread(2, 2000 if batch < 5 else 12000 // batch)
        nlo = max(1, int(nhi * rng.uniform(0.1, 1.0)))
        lo = nhi + rng.choice([0, spread(1, 100000)])
        return _case("", kind, batch, lo, lo + spread(1, 20000), nlo, nhi, rng.choice([0, 0, 5]), **more)
    fmt = rng.choice(["int8", "e4m3"])
    more = dict(hq=hq, hkv=hkv, page=page, fmt=fmt, layout=layout)
    form = rng.choices(["token", "listed", "drafts", "chunk"], [4, 2, 2, 1])[0]
    if form == "chunk":
        batch = rng.choice([1, 1, 2, 3])
        nhi = spread(33, 1000 // batch)
        hi = nhi + spread(1, 15000 // batch)
        return _case("", kind, batch, max(nhi, int(hi * 0.6)), hi, max(1, nhi // 2), nhi, rng.choice([0, 5]), **more)
    batch = spread(1, 64)
    longest = min(1 << 20 if batch == 1 else 131072, 2_000_000 // (batch * hkv))
    hi = spread(min(500, longest), longest)
    lo = max(9, int(hi * rng.uniform(0.1, 1.0)))
    if form == "drafts":
        return _case("", kind, batch, lo, min(hi, 200_000 // batch) + 9, rng.choice([1, 2]), rng.choice([3, 4, 8]), rng.choice([0, 2]), **more) \
            if lo <= 200_000 // batch else _case("", kind, batch, 500, 3000, 1, 4, **more)
    return _case("", kind, batch, lo, hi, budget=rng.choice([256, 700, 1024, 2048]) if form == "listed" else 0, **more)


def _spread(c, lo, hi):
    return [hi - int((i * 0.6180339887498949) % 1.0 * (hi - lo)) for i in range(c["batch"])]


def news(c):
    """New tokens of each request."""
    return _spread(c, c["nlo"], c["nhi"])


def lengths(c):
    """Tokens of each request's sequence, the new ones included."""
    return [max(t, n) for t, n in zip(_spread(c, c["lo"], c["hi"]), news(c))]


def _axis(c):
    """The axis of each rotated pair's frequency: sections, as long as the head's rotated part allows."""
    half = c["rot"] // 2
    return [min(a for a, e in enumerate(FIRST[c["axes"]]) if i * 64 // half < e) for i in range(half)]


def _positions(c, lens, new, total, gen, dev):
    """[axes, rows]: a text token has its place in the sequence on every axis; a request with several tokens and axes shows frames
    whose patches count rows and columns behind the text before them."""
    pos = torch.zeros(c["axes"], total, dtype=torch.int32, device=dev)
    at = 0
    for t, n in zip(lens, new):
        p = torch.arange(t - n, t, device=dev, dtype=torch.int64).repeat(c["axes"], 1)
        if c["axes"] > 1 and n > 1:
            side = max(1, min(32, int(n ** 0.5)))
            i = torch.arange(n, device=dev)
            parts = [i // (side * side), i // side % side, i % side, i][: c["axes"]]
            p = torch.stack(parts) + (t - n)
        pos[:, at:at + n] = p.to(torch.int32)
        at += n
    return pos


def prepare(case, seed):
    c = case
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    s = {"case": c, "gen": gen}
    hq, hkv, B = c["hq"], c["hkv"], c["page"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    half = c["rot"] // 2
    s["inv_freq"] = torch.tensor([BASE ** (-i / half) for i in range(half)], dtype=torch.float32, device=dev)
    s["axis"] = torch.tensor(_axis(c), dtype=torch.int64, device=dev)
    new = news(c)
    if c["kind"] == "rope":
        start = torch.randint(0, 900_000, (c["batch"],), generator=gen, device=dev).tolist()   # long conversations: far positions
        lens = [a + n for a, n in zip(start, new)]
    else:
        lens = lengths(c)
    total = sum(new) + c["pad"]
    s["new"], s["lens"], s["total"] = new, lens, total
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    s["cu"] = torch.tensor(cu, dtype=torch.int32, device=dev)
    s["positions"] = _positions(c, lens, new, total, gen, dev)
    if c["kind"] != "attend":
        if c["fused"]:
            rows = normal(total, (hq + 2 * hkv) * D).to(dt)
            parts = rows.view(total, hq + 2 * hkv, D).split([hq, hkv, hkv], dim=1)
        else:
            parts = [normal(total, h, D).to(dt) for h in (hq, hkv, hkv)]
        s["q"], s["k_new"], s["v_new"] = parts
        s["q_out"] = torch.zeros(total, hq, D, dtype=dt, device=dev)
        s["k_out"] = torch.zeros(total, hkv, D, dtype=dt, device=dev)
    if c["kind"] == "rope":
        if own:
            _handles(s)
        return s
    # the cache: requests whose early pages are all of one shared prefix when nothing reads them (appends), or blocks of their own
    pages = [-(-t // B) for t in lens]
    row = max(pages) + 3
    table = torch.zeros(c["batch"], row, dtype=torch.int32, device=dev)
    shared = 4 if c["kind"] != "attend" else 0
    first = [(t - n) // B if shared else 0 for t, n in zip(lens, new)]
    nb = shared + sum(p - f for p, f in zip(pages, first))
    order = torch.randperm(nb - shared, generator=gen, device=dev).to(torch.int32) + shared
    at = 0
    for b, (p, f) in enumerate(zip(pages, first)):
        if f:
            table[b, :f] = torch.arange(f, device=dev, dtype=torch.int32) % shared
        table[b, f:p] = order[at:at + p - f]
        at += p - f
    s["table"], s["num_blocks"] = table, nb
    s["seq"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    nhd = c["layout"] == "NHD"
    shape = (nb, B, hkv, D) if nhd else (nb, hkv, B, D)

    def heads_first(x):   # a view [block, head, token, dim] of the cache
        return x.transpose(1, 2) if nhd else x

    if c["kind"] == "append":
        for n in ("k", "v"):
            s[n] = heads_first(normal(*shape).to(dt))
    else:
        for n in ("k", "v"):
            codes = torch.empty(shape, dtype=torch.int8 if c["fmt"] == "int8" else torch.float8_e4m3fn, device=dev)
            s[n], s[n + "_scale"] = heads_first(codes), torch.empty(nb, hkv, device=dev)
            offset = 2.0 * normal(hkv, 1, D) if n == "k" else 0.0
            step = max(1, (1 << 27) // (hkv * B * D))
            for p in range(0, nb, step):
                m = min(step, nb - p)
                x = normal(m, hkv, B, D) + offset
                scale = x.abs().amax(dim=(2, 3)) / CODE_MAX[c["fmt"]]
                y = x / scale[:, :, None, None]
                s[n][p:p + m] = y.round().to(torch.int8) if c["fmt"] == "int8" else y.to(torch.float8_e4m3fn)
                s[n + "_scale"][p:p + m] = scale
            s[n + "_tail"] = normal(c["batch"], hkv, B, D) + offset
    if c["kind"] == "attend":
        s["q"] = (2.0 * normal(total, hq, D)).to(dt)   # as peaked as trained heads are
        s["out"] = torch.zeros(total, hq, D, dtype=dt, device=dev)
        s["lse"] = torch.zeros(total, hq, device=dev)
        s["ids"] = s["cnt"] = None
        if c["budget"]:
            # the first page, the last one and a random choice between them, ascending
            k = -(-c["budget"] // B)
            ids = torch.full((c["batch"], hkv, k), -1, dtype=torch.int32, device=dev)
            cnt = torch.zeros(c["batch"], hkv, dtype=torch.int32, device=dev)
            for b, p in enumerate(pages):
                m = min(p, k)
                cnt[b] = m
                key = torch.rand(hkv, p, generator=gen, device=dev)
                key[:, 0] = key[:, -1] = 2.0
                ids[b, :, :m] = key.topk(m, dim=1).indices.sort(dim=1).values.to(torch.int32)
            s["ids"], s["cnt"] = ids, cnt
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a user's program keeps of the library: a context, the rotary description, the view of the cache."""
    import paper_2607_24555_b200 as locks
    from paper_2607_24555_b200.binding import KVQView, KVView, make_config, make_rotary
    c = s["case"]
    row = s["table"].shape[1] if "table" in s else 2
    budget = c["budget"] or 2 * c["page"]
    s["ctx"] = locks.Context(make_config(c["hq"], c["hkv"], 8, "i4" if c["dtype"] == "bf16" else "f32", c["dtype"], c["batch"], row, budget, B=c["page"]),
                             device="cuda:0")
    s["rotary"] = make_rotary(s["inv_freq"].tolist(), axis=s["axis"].tolist(), interleaved=c["inter"])
    if c["kind"] == "append":
        s["kv"] = KVView(s["k"], s["v"], s["k"].stride()[:3], s["num_blocks"], s["table"], s["seq"])
    elif c["kind"] != "rope":
        s["kv"] = KVQView(s["k"], s["v"], s["k_scale"], s["v_scale"], s["k_tail"], s["v_tail"], s["table"], s["seq"])
    # a token per request needs no offsets, unless rows behind them belong to nobody
    s["own_cu"] = s["cu"] if c["nhi"] > 1 or c["pad"] else None


def _outputs(s):
    kind = s["case"]["kind"]
    if kind == "rope":
        return {"q": s["q_out"], "k": s["k_out"]}
    if kind == "append":
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    if kind == "qappend":
        return {n: s[n] for n in ("q_out", "k", "v", "k_scale", "v_scale", "k_tail", "v_tail")}
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    s = state
    kind = s["case"]["kind"]
    if own:
        ctx, batch = s["ctx"], s["case"]["batch"]
        if kind == "rope":
            ctx.locks_rope(s["rotary"], s["positions"], s["q"], s["q_out"], s["k_new"], s["k_out"])
        elif kind == "append":
            ctx.locks_append_rows(s["k_new"], s["v_new"], s["kv"], batch, rotary=s["rotary"], positions=s["positions"], q=s["q"],
                             q_out=s["q_out"], cu_tokens=s["own_cu"])
        elif kind == "qappend":
            ctx.locks_kvq_append(s["k_new"], s["v_new"], s["kv"], batch, rotary=s["rotary"], positions=s["positions"], q=s["q"],
                                 q_out=s["q_out"], cu_tokens=s["own_cu"])
        else:
            ctx.locks_kvq_attend(s["q"], s["kv"], batch, s["out"], lse=s["lse"], page_ids=s["ids"], page_count=s["cnt"],
                                 cu_tokens=s["own_cu"])
    elif kind == "rope":
        s["q_out"].copy_(_rotate(s, s["q"]))
        s["k_out"].copy_(_rotate(s, s["k_new"]))
    elif kind == "append":
        _plain_append(s)
    elif kind == "qappend":
        _plain_qappend(s)
    else:
        _plain_attend(s)
    return _outputs(s)


# ------------------------------------------------------------------------------------------------ plain forms
def _rotate(s, x):
    """x [rows, heads, D] rotated, in 32 bits; the angles in 64."""
    c = s["case"]
    half = c["rot"] // 2
    angle = s["positions"][s["axis"]].double() * s["inv_freq"].double()[:, None]   # [half, rows]
    cos, sin = angle.cos().float().T[:, None], angle.sin().float().T[:, None]
    y = x.float().clone()
    a, b = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["inter"] else (slice(0, half), slice(half, c["rot"]))
    xa, xb = x[..., a].float(), x[..., b].float()
    y[..., a] = xa * cos - xb * sin
    y[..., b] = xa * sin + xb * cos
    return y


def _tokens(s):
    """Request and place in its sequence of each row that belongs to a request."""
    cu, seq = s["cu"].long(), s["seq"].long()
    row = torch.arange(sum(s["new"]), device=cu.device)
    req = torch.bucketize(row, cu[1:], right=True)
    return req, seq[req] - cu[req + 1] + row


def _plain_append(s):
    B = s["case"]["page"]
    req, pos = _tokens(s)
    n = len(req)
    s["q_out"][:n] = _rotate(s, s["q"])[:n].to(s["q_out"].dtype)
    block = s["table"].long()[req, pos // B]
    s["k"][block, :, pos % B] = _rotate(s, s["k_new"])[:n].to(s["k"].dtype)
    s["v"][block, :, pos % B] = s["v_new"][:n]


def _plain_qappend(s):
    """Windows of whole pages per request, from the first page that gets a token on: its earlier tokens from the tail."""
    c = s["case"]
    B, dev = c["page"], s["seq"].device
    n = sum(s["new"])
    k_rows, v_rows = _rotate(s, s["k_new"]), s["v_new"].float()
    s["q_out"][:n] = _rotate(s, s["q"])[:n].to(s["q_out"].dtype)
    seq, cu = s["seq"].long(), s["cu"].long()
    start = seq - (cu[1:] - cu[:-1])
    p0, done = start // B, seq // B
    most = max(-(-t // B) - (t - m) // B for t, m in zip(s["lens"], s["new"]))
    pos = (p0 * B)[:, None] + torch.arange(most * B, device=dev)
    from_tail = (pos < start[:, None])[:, :, None, None]
    row = (cu[:-1, None] + pos - start[:, None]).clamp(0, s["total"] - 1)
    page = p0[:, None] + torch.arange(most, device=dev)
    complete = page < done[:, None]
    block = s["table"].long().gather(1, page.clamp(max=s["table"].shape[1] - 1))[complete]
    last = (done * B)[:, None] + torch.arange(B, device=dev)   # places of the unfinished page
    fresh = ((last >= start[:, None]) & (last < seq[:, None]))[:, None, :, None]
    last_row = (cu[:-1, None] + last - start[:, None]).clamp(0, s["total"] - 1)
    b = torch.arange(c["batch"], device=dev)[:, None]
    for name, rows in (("k", k_rows), ("v", v_rows)):
        tail = s[name + "_tail"]
        x = torch.where(from_tail, tail[b, :, pos % B], rows[row])
        x = x.unflatten(1, (most, B)).transpose(2, 3)[complete]   # [pages, hkv, B, D]
        amax = x.abs().amax(dim=(2, 3))
        scale = torch.where(amax >= TINY, amax / CODE_MAX["e4m3"], 0.0)
        y = torch.where(scale[:, :, None, None] > 0, x / scale[:, :, None, None], 0.0)
        s[name][block] = y.to(torch.float8_e4m3fn)
        s[name + "_scale"][block] = scale
        tail.copy_(torch.where(fresh, rows[last_row].transpose(1, 2), tail))


def _plain_attend(s):
    c = s["case"]
    B, hkv, g, dev = c["page"], c["hkv"], c["hq"] // c["hkv"], s["seq"].device
    seq, cu = s["seq"].long(), s["cu"].long()
    if s["ids"] is None:
        most = max(-(-t // B) for t in s["lens"])
        page = torch.arange(most, device=dev).expand(c["batch"], 1, most)
        block = s["table"].long()[:, None, :most]
    else:
        page = s["ids"].long()
        block = s["table"].long()[:, None].expand(-1, hkv, -1).gather(2, page.clamp(min=0))
    head = torch.arange(hkv, device=dev)[None, :, None]
    here = (page >= 0) & (page < seq[:, None, None] // B)   # finished pages; the unfinished one is in the tail
    pos = (page[..., None] * B + torch.arange(B, device=dev)).flatten(2)   # [batch, 1 or hkv, tokens]
    pos = torch.where((page >= 0).repeat_interleave(B, dim=2), pos, 1 << 40)
    unfinished = (page == seq[:, None, None] // B).expand(-1, hkv, -1)
    kv = []
    for name in ("k", "v"):
        x = s[name][block, head].float() * s[name + "_scale"][block, head][..., None, None]
        x = torch.where(here.expand(-1, hkv, -1)[..., None, None], x, 0.0)
        x = torch.where(unfinished[..., None, None], s[name + "_tail"][:, :, None], x)
        kv.append(x.flatten(2, 3))   # [batch, hkv, tokens, D]
    m = max(s["new"])
    j = torch.arange(m, device=dev)
    live = j < (cu[1:] - cu[:-1])[:, None]
    row = (cu[:-1, None] + j).clamp(max=s["total"] - 1)
    limit = seq[:, None] - (cu[1:] - cu[:-1])[:, None] + j + 1   # tokens that row j of a request sees
    q = s["q"].float()[row].unflatten(2, (hkv, g)).permute(0, 2, 1, 3, 4).flatten(2, 3)   # [batch, hkv, m g, D]
    score = (q @ kv[0].transpose(2, 3)) * (D ** -0.5)
    seen = pos[:, :, None, :] < limit.repeat_interleave(g, dim=1)[:, None, :, None]
    score = score.masked_fill_(~seen, -math.inf)
    top = score.amax(dim=3, keepdim=True)
    p = (score - top).exp_()
    total = p.sum(dim=3, keepdim=True)
    out = ((p @ kv[1]) / total).unflatten(2, (m, g)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    lse = (top + total.log()).squeeze(3).unflatten(2, (m, g)).permute(0, 2, 1, 3).flatten(2)
    s["out"][row[live]] = out[live].to(s["out"].dtype)
    s["lse"][row[live]] = lse[live]


# ------------------------------------------------------------------------------------------------ 64 bits
def _turned(s, x):
    """Rows rotated as complex numbers in 64 bits: a pair of dimensions is one number, times e^(i angle)."""
    c = s["case"]
    pos = s["positions"].double()
    w = s["inv_freq"].double()
    phase = torch.stack([pos[a] * f for a, f in zip(s["axis"].tolist(), w)], dim=-1)[:, None]   # [rows, 1, half]
    x = x.double()
    r, rest = x[..., :c["rot"]], x[..., c["rot"]:]
    pairs = r.unflatten(-1, (c["rot"] // 2, 2)) if c["inter"] else r.unflatten(-1, (2, c["rot"] // 2)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(phase), phase)
    back = torch.view_as_real(z)
    back = back if c["inter"] else back.transpose(-1, -2)
    return torch.cat([back.flatten(-2), rest], dim=-1)


def _e4m3(x):
    """Nearest number of four exponent and three fraction bits, ties to even, at most 448."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -40))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = case, case["kind"]
    B, n = c["page"], sum(s["new"])
    if kind == "rope":
        return {"q": _turned(s, s["q"]), "k": _turned(s, s["k_new"])}
    if kind == "append":
        q = s["q_out"].double()
        q[:n] = _turned(s, s["q"])[:n]
        got = {"q": q, "k": s["k"].double(), "v": s["v"].double()}
        rows = {"k": _turned(s, s["k_new"]), "v": s["v_new"].double()}
        at = 0
        for b, (t, m) in enumerate(zip(s["lens"], s["new"])):
            place = torch.arange(t - m, t, device=q.device)
            block = s["table"][b].long()[place // B]
            for name in ("k", "v"):
                got[name][block, :, place % B] = rows[name][at:at + m]
            at += m
        return got
    if kind == "qappend":
        got = {x: s[x].double() for x in ("q_out", "k", "v", "k_scale", "v_scale", "k_tail", "v_tail")}
        got["q_out"][:n] = _turned(s, s["q"])[:n]
        rows = {"k": _turned(s, s["k_new"]), "v": s["v_new"].double()}
        at = 0
        for b, (t, m) in enumerate(zip(s["lens"], s["new"])):
            before = (t - m) % B
            whole = t // B - (t - m) // B
            blocks = s["table"][b].long()[(t - m) // B:t // B]
            for name in ("k", "v"):
                x = rows[name][at:at + m].transpose(0, 1)                               # [hkv, m, D]
                x = torch.cat([got[name + "_tail"][b, :, :before], x], dim=1)
                if whole:
                    y = x[:, :whole * B].unflatten(1, (whole, B)).transpose(0, 1)       # [whole, hkv, B, D]
                    top = y.abs().flatten(2).amax(2)
                    scale = top / 448.0 * (top >= TINY)
                    got[name][blocks] = _e4m3(y / scale.clamp(min=1e-300)[..., None, None]) * (scale > 0)[..., None, None]
                    got[name + "_scale"][blocks] = scale
                rest = x[:, whole * B:]
                got[name + "_tail"][b, :, :rest.shape[1]] = rest
            at += m
        return got
    out, lse = s["out"].double(), s["lse"].double()
    g = c["hq"] // c["hkv"]
    at = 0
    for b, (t, m) in enumerate(zip(s["lens"], s["new"])):
        for h in range(c["hkv"]):
            pages = torch.arange(-(-t // B), device=out.device) if s["ids"] is None else s["ids"][b, h, :int(s["cnt"][b, h])].long()
            blocks = s["table"][b].long()[pages]
            x = {}
            for name in ("k", "v"):
                y = s[name][blocks, h].double() * s[name + "_scale"][blocks, h].double()[:, None, None]
                y[pages == t // B] = s[name + "_tail"][b, h].double()
                x[name] = y.flatten(0, 1)
            place = (pages[:, None] * B + torch.arange(B, device=out.device)).flatten()
            x, place = {name: y[place < t] for name, y in x.items()}, place[place < t]
            q = s["q"][at:at + m, h * g:(h + 1) * g].double()
            step = max(1, (1 << 27) // (g * max(1, len(place))))
            for i in range(0, m, step):
                score = q[i:i + step] @ x["k"].T / math.sqrt(D)                          # [rows, g, tokens]
                limit = t - m + 1 + torch.arange(i, min(i + step, m), device=out.device)
                score.masked_fill_((place >= limit[:, None])[:, None], -math.inf)
                out[at + i:at + i + step, h * g:(h + 1) * g][: len(limit)] = torch.softmax(score, -1) @ x["v"]
                lse[at + i:at + i + step, h * g:(h + 1) * g][: len(limit)] = torch.logsumexp(score, -1)
        at += m
    return {"out": out, "lse": lse}


def work(case):
    c = case
    esz, hq, hkv, B = 2 if c["dtype"] == "bf16" else 4, c["hq"], c["hkv"], c["page"]
    n = sum(news(c))
    turn = 3 * c["rot"] * n
    if c["kind"] == "rope":
        return {"bytes": n * (2 * (hq + hkv) * D * esz + 4 * c["axes"]), "flops": turn * (hq + hkv)}
    if c["kind"] == "append":
        return {"bytes": n * (2 * (hq + 2 * hkv) * D * esz + 4 * c["axes"] + 4), "flops": turn * (hq + hkv)}
    if c["kind"] == "qappend":
        byts, flops = n * ((2 * hq + 2 * hkv) * D * esz + 4 * c["axes"] + 4), turn * (hq + hkv)
        for t, m in zip(lengths(c), news(c)):
            whole = t // B - (t - m) // B
            byts += whole * hkv * 2 * (B * D + 4)
            if whole:
                byts += (t - m) % B * hkv * D * 8   # what the tail held of the first of them
            byts += min(m, t % B) * hkv * D * 8
            flops += whole * hkv * 2 * B * D * 3
        return {"bytes": byts, "flops": flops}
    byts, flops = n * hq * (2 * D * esz + 4), 0
    for t, m in zip(lengths(c), news(c)):
        pages = -(-t // B)
        if c["budget"]:
            k = -(-c["budget"] // B)
            read = t - max(0, pages - k) * B
            byts += 4 * hkv * min(k, pages)
        else:
            read = t
        rest = t % B
        byts += hkv * ((read - rest) * 2 * D + (read - rest) // B * 8 + rest * 8 * D) + 4 * min(pages, -(-read // B))
        flops += 4 * hq * D * sum(read - i for i in range(m))
    return {"bytes": byts, "flops": flops}
