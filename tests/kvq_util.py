"""Plain 64-bit forms of the calls around a decode step (rotary positions, appends, the 8-bit cache) and random caches for them."""
import math

import numpy as np
import torch

D = 128
CODE_MAX = {"int8": 127.0, "e4m3": 448.0}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def f64(t):
    return t.detach().to("cpu").to(torch.float64)


def cu_of(new, dev="cpu"):
    return torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device=dev)


def rotate(x, pos, inv_freq, axis=None, interleaved=False):
    """x [rows, heads, D] (64 bits), pos [axes, rows] ints, inv_freq fp32 values."""
    half = len(inv_freq)
    y = x.clone()
    for i in range(half):
        a = 0 if axis is None else axis[i]
        ang = pos[a].to(torch.float64) * float(np.float32(inv_freq[i]))
        c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[:, :, p] = x[:, :, p] * c - x[:, :, q] * s
        y[:, :, q] = x[:, :, p] * s + x[:, :, q] * c
    return y


def turn_bound(x, half, interleaved):
    """What fp32 arithmetic may be off, per element: sine and cosine within 2^-22 each (two units, of 2^-23 at most) and an angle
    within 2^-23 (a fraction of a turn rounded to fp32, times pi); two products and a sum rounded: 2^-23 more."""
    y = torch.zeros_like(x)
    m = x.abs()
    for i in range(half):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[:, :, p] = y[:, :, q] = (m[:, :, p] + m[:, :, q]) * (2.0 ** -22 + 2.0 ** -22 + 2.0 ** -23)
    return y


def e4m3(x):
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -40))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def value_step(x, scale, fmt):
    """Half a step of the format around x, scale given."""
    if fmt == "int8":
        return torch.full_like(x, 0.5) * scale
    return torch.maximum(x.abs() * 2.0 ** -4, 2.0 ** -10 * scale * torch.ones_like(x))


def random_cache(gen, batch, lens, Hkv, B, fmt, layout="HND", rows_more=2, spare=3, k_offset=2.0, dev="cuda:0", spread=0.0):
    """An 8-bit cache of random pages, with tails, permuted blocks and a block table whose unused entries lie outside the cache."""
    from paper_2607_24555_b200 import new_kvq_cache
    pages = [-(-t // B) for t in lens]
    nb = sum(pages) + spare
    order = torch.randperm(nb, generator=gen)
    table = torch.full((batch, max(pages) + rows_more), 1 << 30, dtype=torch.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = order[at:at + p].to(torch.int32)
        at += p
    seq = torch.tensor(lens, dtype=torch.int32)
    kvq = new_kvq_cache(nb, batch, Hkv, B, table.to(dev), seq.to(dev), fmt=fmt, layout=layout)
    for n, off in (("k", k_offset), ("v", 0.0)):
        x = torch.randn(nb, Hkv, B, D, generator=gen) + off * torch.randn(1, Hkv, 1, D, generator=gen)
        x = x * torch.exp(spread * torch.randn(nb, Hkv, 1, 1, generator=gen))
        scale = x.abs().amax(dim=(2, 3)) / CODE_MAX[fmt]
        y = x / scale[:, :, None, None]
        codes = y.round().to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)
        getattr(kvq, n).copy_(codes.to(dev))
        getattr(kvq, n + "_scale").copy_(scale.to(dev))
        getattr(kvq, n + "_tail").copy_((torch.randn(batch, Hkv, B, D, generator=gen) + off).to(dev))
    return kvq


def sequence(kvq, b, h, T, B, pages=None):
    """Keys and values (64 bits) that request b's KV head h holds in `pages` (None: all), with their places."""
    pages = list(range(-(-T // B))) if pages is None else pages
    ks, vs, pos = [], [], []
    for p in pages:
        m = min(B, T - p * B)
        if m <= 0:
            continue
        if (p + 1) * B <= T:
            blk = int(kvq.block_table[b, p])
            ks.append(f64(kvq.k[blk, h].float()) * f64(kvq.k_scale[blk, h]))
            vs.append(f64(kvq.v[blk, h].float()) * f64(kvq.v_scale[blk, h]))
        else:
            ks.append(f64(kvq.k_tail[b, h, :m]))
            vs.append(f64(kvq.v_tail[b, h, :m]))
        pos.append(torch.arange(p * B, p * B + m))
    if not ks:
        return torch.zeros(0, D, dtype=torch.float64), torch.zeros(0, D, dtype=torch.float64), torch.zeros(0, dtype=torch.int64)
    return torch.cat(ks), torch.cat(vs), torch.cat(pos)


def attend(q, kvq, lens, new, Hkv, B, ids=None, cnt=None, per_head=False):
    """(out, lse, bound): 64-bit attention, and what the kernel may be off by: its result's rounding to bf16 (2^-8 of it); weights in
    fp16 (2^-11 of each, 2^-25 at least: below fp16's normal numbers); the unfinished page's elements in fp16 (2^-11 of each, in the
    scores and in the values); scores summed in fp32 (128 products, each sum within 2^-23: 2^-16 of the sum of magnitudes).
    The few-token form multiplies weights by code + 128 (up to 255, times the page's scale) and takes 128 sum of weights off in the same
    accumulator: 16 products and a start, each cut off at 2^-23 of the largest, which is at most 255 times its weight: so a
    tile's sum is off by at most 17 x 255 x 2^-23 of weight times scale, which no small output makes smaller.  (Seen: a token of
    weight 0.9988 whose code is 0, others' values adding up to 8.2e-5 and off by 1.6e-6, with 17 x 255 x 2^-23 x 0.024 = 1.2e-5.)"""
    n, Hq = q.shape[0], q.shape[1]
    G = Hq // Hkv
    out, lse = torch.zeros(n, Hq, D, dtype=torch.float64), torch.full((n, Hq), -math.inf, dtype=torch.float64)
    bound, lse_bound = torch.zeros(n, Hq, D, dtype=torch.float64), torch.zeros(n, Hq, dtype=torch.float64)
    q64, sm = f64(q), D ** -0.5
    row = 0
    for b, (T, m) in enumerate(zip(lens, new)):
        for hh in range(Hq if per_head else Hkv):
            h, heads = (hh // G, slice(hh, hh + 1)) if per_head else (hh, slice(hh * G, hh * G + G))
            pages = None if ids is None else [int(p) for p in ids[b, hh, :int(cnt[b, hh])]]
            k, v, pos = sequence(kvq, b, h, T, B, pages)
            vs = torch.tensor([0.0 if int(i) >= T // B * B else float(kvq.v_scale[int(kvq.block_table[b, int(i) // B]), h]) for i in pos[::16]],
                              dtype=torch.float64).repeat_interleave(16)[:len(pos)]
            if m == 0 or len(pos) == 0:
                continue
            qq = q64[row:row + m, heads]                                  # [m, g, D]
            see = (pos[None] < (T - m + 1 + torch.arange(m))[:, None])    # [m, tokens]
            some = see.any(1)
            s = (qq @ k.T * sm).masked_fill(~see[:, None], -math.inf)
            ll = torch.logsumexp(s, 2)
            p = torch.exp(s - ll.masked_fill(~some[:, None], 0.0)[..., None])
            o = p @ v
            mag = (qq.abs() @ k.abs().T) * sm
            tail = (pos >= T // B * B).to(torch.float64)
            d = mag * (2.0 ** -16 + tail * 2.0 ** -11) + 2.0 ** -20       # of a score; and of the exponential
            pd = p * torch.expm1(d)
            w = pd @ v.abs() + pd.sum(2, keepdim=True) * o.abs()
            top = s.max(2).values
            low = 2.0 ** -25 * torch.exp(torch.where(some[:, None], top - ll, 0.0))[..., None] * (see.to(torch.float64) @ v.abs())[:, None]
            err = 2.0 ** -8 * o.abs() + 1.01 * (w + 2.0 ** -11 * (p @ v.abs()) + 2.0 ** -11 * ((p * tail) @ v.abs()) + low) + 17 * 255 * 2.0 ** -23 * (p @ vs)[..., None] + 1e-30
            lerr = (p * d).sum(2) + 2.0 ** -20 * (1 + ll.abs())
            sel = some.nonzero()[:, 0]
            out[row + sel, heads], lse[row + sel, heads] = o[sel], ll[sel]
            bound[row + sel, heads], lse_bound[row + sel, heads] = err[sel], lerr[sel]
        row += m
    return out, lse, bound, lse_bound
