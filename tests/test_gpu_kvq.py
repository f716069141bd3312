"""Rotary positions, appends and the 8-bit cache on the GPU, against plain 64-bit forms (kvq_util.py)."""
import math

import numpy as np
import pytest
import torch

import kvq_util as U
import paper_2607_24555_b200 as locks
from paper_2607_24555_b200.binding import KVView, make_config, make_rotary, new_kvq_cache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def context(Hq, Hkv, B=16, batch=8, pages=64, budget=64, dtype="bf16", **kw):
    return locks.Context(make_config(Hq, Hkv, 8, "i4" if dtype == "bf16" else "f32", dtype, batch, pages, budget, B=B, **kw), device=DEV)


def freqs(rot, base=10000.0):
    return [float(np.float32(base ** (-2 * i / rot))) for i in range(rot // 2)]


def rows(gen, n, heads, dtype, fused=False):
    if not fused:
        return torch.randn(n, heads, 128, generator=gen).to(DT[dtype]).to(DEV)
    return torch.randn(n, heads + 3, 128, generator=gen).to(DT[dtype]).to(DEV)[:, 2:2 + heads]


def near(got, want, bound, what):
    got = U.f64(got)
    assert not torch.isnan(got).any(), what
    over = (got - want).abs() - bound
    assert float(over.max()) <= 0, (what, float(over.max()), float((got - want).abs().max()))


# ------------------------------------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,Hkv,rot,axes,fused", [(1, 4, 1, 128, 1, False), (7, 28, 4, 96, 3, True), (33, 40, 8, 16, 4, False), (130, 5, 5, 112, 2, True)])
def test_rope(n, Hq, Hkv, rot, axes, fused, dtype, inter):
    gen = torch.Generator().manual_seed(n)
    ctx = context(Hq, Hkv, dtype=dtype)
    f = freqs(rot)
    axis = [i % axes for i in range(rot // 2)]
    pos = torch.randint(-5, 1 << 20, (axes, n), generator=gen, dtype=torch.int32)
    q, k = rows(gen, n, Hq, dtype, fused), rows(gen, n, Hkv, dtype, fused)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    ctx.locks_rope(make_rotary(f, axis, inter), pos.to(DEV), q, qo, k, ko)
    for x, y in ((q, qo), (k, ko)):
        want = U.rotate(U.f64(x), pos, f, axis, inter)
        turned = U.turn_bound(U.f64(x), rot // 2, inter)
        near(y, want, turned + U.HALF_STEP[dtype] * (want.abs() + turned), "rope")
        assert torch.equal(y[..., rot:], x[..., rot:])
    want = qo.clone()
    ctx.locks_rope(make_rotary(f, axis, inter), pos.to(DEV), q, q)   # in place, queries alone
    assert torch.equal(q, want)
    ctx.locks_rope(make_rotary(f, axis, inter), pos.to(DEV), None, None, k, k)
    assert torch.equal(k, ko)


def test_rope_keeps_far_positions_apart():
    """Two positions a million apart whose difference is all that a score depends on."""
    ctx = context(4, 4, dtype="f32")
    f = freqs(128)
    gen = torch.Generator().manual_seed(0)
    x = rows(gen, 2, 4, "f32")
    x[1] = x[0]
    out = torch.empty_like(x)
    dots = []
    for base in (0, 1 << 20, (1 << 30) - 7):
        ctx.locks_rope(make_rotary(f), torch.tensor([base, base + 5], dtype=torch.int32, device=DEV), x, out)
        y = U.f64(out)
        dots.append((y[0] * y[1]).sum(-1))
    scale = float((U.f64(x[0]) ** 2).sum(-1).max())
    # every term's two factors are within 2^-21 of their pair's magnitude, and a pair has two terms
    for d in dots[1:]:
        assert float((d - dots[0]).abs().max()) <= 8 * 2.0 ** -21 * scale


# ------------------------------------------------------------------------------------------------ appends, cache in the type of the rows
@pytest.mark.parametrize("dtype,B,layout", [("bf16", 16, "HND"), ("bf16", 32, "NHD"), ("f32", 64, "HND"), ("f32", 16, "NHD")])
@pytest.mark.parametrize("lens,new,pad,given", [([1, 17, 400], [1, 1, 1], 0, False), ([40, 33, 200, 7, 16], [40, 1, 0, 7, 16], 3, True), ([129], [129], 0, False)])
def test_append_rows(lens, new, pad, given, dtype, B, layout):
    Hq, Hkv, batch, n = 6, 3, len(lens), sum(new) + pad
    gen = torch.Generator().manual_seed(n + B)
    ctx = context(Hq, Hkv, B=B, batch=batch, pages=30, budget=2 * B, dtype=dtype)
    pages = [-(-t // B) for t in lens]
    table = torch.full((batch, 30), -1, dtype=torch.int32)
    perm = torch.randperm(sum(pages) + 2, generator=gen).to(torch.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = perm[at:at + p]
        at += p
    shape = (sum(pages) + 2, Hkv, B, 128) if layout == "HND" else (sum(pages) + 2, B, Hkv, 128)
    caches = [torch.randn(shape, generator=gen).to(DT[dtype]).to(DEV) for _ in range(2)]
    kc, vc = [c if layout == "HND" else c.transpose(1, 2) for c in caches]
    want = [U.f64(kc), U.f64(vc)]
    kv = KVView(kc, vc, kc.stride()[:3], shape[0], table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV))
    q, k, v = rows(gen, n, Hq, dtype, True), rows(gen, n, Hkv, dtype), rows(gen, n, Hkv, dtype, True)
    qo = torch.full((n, Hq, 128), 7.0, dtype=DT[dtype], device=DEV)
    f = freqs(64)
    pos = torch.randint(0, 5000, (2, n), generator=gen, dtype=torch.int32) if given else None
    axis = [i % 2 for i in range(32)] if given else None
    use_cu = pad or max(new) > 1
    ctx.locks_append_rows(k, v, kv, batch, rotary=make_rotary(f, axis), positions=None if pos is None else pos.to(DEV), q=q, q_out=qo,
                          cu_tokens=U.cu_of(new, DEV) if use_cu else None)
    place = torch.cat([torch.arange(t - m, t) for t, m in zip(lens, new)])
    live = sum(new)
    p = torch.cat([place, torch.zeros(pad, dtype=torch.int64)])[None] if pos is None else pos
    bound = torch.zeros_like(want[0])
    turned = U.rotate(U.f64(k), p, f, axis)
    half = U.HALF_STEP[dtype]
    tb = U.turn_bound(U.f64(k), 32, False)
    i = 0
    for b, (t, m) in enumerate(zip(lens, new)):
        for at in range(t - m, t):
            blk = int(table[b, at // B])
            want[0][blk, :, at % B] = turned[i]
            bound[blk, :, at % B] = tb[i] + half * (turned[i].abs() + tb[i])
            want[1][blk, :, at % B] = U.f64(v[i])
            i += 1
    near(kc, want[0], bound, "keys")
    assert torch.equal(U.f64(vc), want[1])
    wq = U.rotate(U.f64(q), p, f, axis)
    tq = U.turn_bound(U.f64(q), 32, False)
    near(qo[:live], wq[:live], (tq + half * (wq.abs() + tq))[:live], "queries")
    assert bool((qo[live:] == 7.0).all()), "rows behind the last request"
    assert ctx.locks_poll_status() == 0
    # without rotation: the rows as they are
    ctx.locks_append_rows(k, v, kv, batch, cu_tokens=U.cu_of(new, DEV) if use_cu else None)
    i = 0
    for b, (t, m) in enumerate(zip(lens, new)):
        for at in range(t - m, t):
            assert torch.equal(kc[int(table[b, at // B]), :, at % B], k[i])
            i += 1


def test_append_rows_skips_what_is_not_there():
    """A place beyond the table's row, a block outside the cache and a request shorter than its new tokens are reported and skipped; a
    request of length zero has no token."""
    ctx = context(4, 2, batch=4, pages=2)
    gen = torch.Generator().manual_seed(3)
    cache = [torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    table = torch.tensor([[0, 1], [2, 1 << 30], [3, 3], [-1, -1]], dtype=torch.int32, device=DEV)
    k, v = rows(gen, 4, 2, "bf16"), rows(gen, 4, 2, "bf16")

    def run(lens):
        for c in cache:
            c.zero_()
        ctx.locks_append_rows(k, v, KVView(*cache, cache[0].stride()[:3], 4, table, torch.tensor(lens, dtype=torch.int32, device=DEV)), 4)
        return ctx.locks_poll_status(), cache[0].abs().sum((1, 2, 3)).cpu()

    st, used = run([1, 5, 0, 0])
    assert st == 0 and list(used > 0) == [True, False, True, False]
    st, used = run([33, 16, 16, 0])      # 33 tokens do not fit a row of 32
    assert st == -6 and list(used > 0) == [False, False, True, True]
    st, used = run([32, 17, 0, 0])       # block 1 << 30
    assert st == -6 and list(used > 0) == [False, True, False, False]
    st, used = run([-3, 1, 1, 1])        # request 3: block -1
    assert st == -6 and list(used > 0) == [False, False, True, True]


# ------------------------------------------------------------------------------------------------ appends, 8-bit cache
def check_page(kvq, name, blk, h, x, fmt, tol, what):
    """x [B, D]: the page's values in 64 bits, right to tol."""
    got = U.f64(getattr(kvq, name)[blk, h].float())
    scale = float(getattr(kvq, name + "_scale")[blk, h])
    amax = float(x.abs().max())
    if amax < 2.0 ** -100:
        assert scale == 0 and not bool(got.any()), what
        return
    ref = amax / U.CODE_MAX[fmt]
    at = (x.abs() == amax)
    assert abs(scale - ref) <= ref * 2.0 ** -23 + float((tol * at).max()) / U.CODE_MAX[fmt] + float(tol.max()) / U.CODE_MAX[fmt], what
    # a quotient's rounding to fp32 moves a code only at a border, where both neighbours are half a step away
    off = (got * scale - x).abs() - (U.value_step(x, scale, fmt) * (1 + 2.0 ** -20) + tol * (1 + 2.0 ** -4) + scale * 448 * 2.0 ** -22)
    assert float(off.max()) <= 0, (what, float(off.max()))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("B,layout,inter", [(16, "HND", False), (16, "NHD", True), (32, "HND", False), (64, "NHD", False)])
@pytest.mark.parametrize("Hq,Hkv,lens,new,pad", [
    (4, 2, [1, 16, 17, 400], [1, 1, 1, 1], 0),
    (28, 4, [100, 33, 200, 7, 64, 130], [100, 1, 0, 7, 33, 130], 5),
    (5, 5, [643], [300], 0)])
def test_kvq_append(Hq, Hkv, lens, new, pad, B, layout, inter, fmt):
    batch, n = len(lens), sum(new) + pad
    gen = torch.Generator().manual_seed(n + B)
    kvq = U.random_cache(gen, batch, lens, Hkv, B, fmt, layout)
    ctx = context(Hq, Hkv, B=B, batch=batch, pages=kvq.block_table.shape[1], budget=2 * B)
    before = {x: getattr(kvq, x).clone() for x in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail")}
    q, k, v = rows(gen, n, Hq, "bf16", True), rows(gen, n, Hkv, "bf16", True), rows(gen, n, Hkv, "bf16")
    qo = torch.full((n, Hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    f, axes = freqs(128), 3
    axis = [0] * 16 + [1] * 24 + [2] * 24
    pos = torch.randint(0, 70000, (axes, n), generator=gen, dtype=torch.int32)
    ctx.locks_kvq_append(k, v, kvq, batch, rotary=make_rotary(f, axis, inter), positions=pos.to(DEV), q=q, q_out=qo,
                         cu_tokens=U.cu_of(new, DEV) if pad or max(new) > 1 else None)
    assert ctx.locks_poll_status() == 0
    live = sum(new)
    wq, tq = U.rotate(U.f64(q), pos, f, axis, inter), U.turn_bound(U.f64(q), 64, inter)
    near(qo[:live], wq[:live], (tq + 2.0 ** -8 * (wq.abs() + tq))[:live], "queries")
    assert bool((qo[live:] == 7.0).all())
    rowsk, tolk = U.rotate(U.f64(k), pos, f, axis, inter), U.turn_bound(U.f64(k), 64, inter)
    touched = set()
    at = 0
    for b, (t, m) in enumerate(zip(lens, new)):
        start = t - m
        for name, x, tol in (("k", rowsk, tolk), ("v", U.f64(v), torch.zeros_like(tolk))):
            tail = U.f64(before[name + "_tail"][b])
            w0 = start // B * B
            whole = torch.cat([tail[:, :start - w0], x[at:at + m].transpose(0, 1)], 1)
            wt = torch.cat([torch.zeros_like(tail[:, :start - w0]), tol[at:at + m].transpose(0, 1)], 1)
            if m == 0:
                assert torch.equal(getattr(kvq, name + "_tail")[b], before[name + "_tail"][b])
                continue
            for p in range(start // B, t // B):
                blk = int(kvq.block_table[b, p])
                touched.add(blk)
                for h in range(Hkv):
                    o = p * B - w0
                    check_page(kvq, name, blk, h, whole[h, o:o + B], fmt, wt[h, o:o + B], (name, b, p, h))
            got, last = U.f64(getattr(kvq, name + "_tail")[b]), t // B * B
            if last >= w0:
                for i in range(max(last, start), t):
                    near(got[:, i - last], whole[:, i - w0], wt[:, i - w0] * 1.0001 + 2.0 ** -24 * whole[:, i - w0].abs(), "tail")
                if last == w0:   # the page was unfinished and is: its old tokens stay, and what lies behind them too
                    assert torch.equal(got[:, :start - last], tail[:, :start - last])
                assert torch.equal(got[:, t - last:], tail[:, t - last:])
        at += m
    rest = [i for i in range(kvq.k.shape[0]) if i not in touched]
    for x in ("k", "v", "k_scale", "v_scale"):
        a, c = getattr(kvq, x)[rest].float(), before[x][rest].float()
        assert torch.equal(a, c), x


def test_kvq_append_does_not_depend_on_how_a_prompt_is_cut():
    Hq, Hkv, T = 4, 2, 150
    gen = torch.Generator().manual_seed(1)
    q, k, v = rows(gen, T, Hq, "bf16"), rows(gen, T, Hkv, "bf16"), rows(gen, T, Hkv, "bf16")
    rot = make_rotary(freqs(128))
    got = []
    for B in (16, 64):
        for cuts in ([150], [1] * 150, [17, 3, 100, 30]):
            table = torch.arange(10, dtype=torch.int32, device=DEV)[None]
            kvq = new_kvq_cache(10, 1, Hkv, B, table, torch.zeros(1, dtype=torch.int32, device=DEV))
            ctx = context(Hq, Hkv, B=B, batch=1, pages=10, budget=2 * B)
            qo, at = torch.empty_like(q), 0
            for m in cuts:
                kvq.seq_lens += m
                ctx.locks_kvq_append(k[at:at + m], v[at:at + m], kvq, 1, rotary=rot, q=q[at:at + m], q_out=qo[at:at + m],
                                     cu_tokens=torch.tensor([0, m], dtype=torch.int32, device=DEV))
                at += m
            n = T % B
            got.append((B, qo.clone(), kvq.k.clone(), kvq.v.clone(), kvq.k_scale.clone(), kvq.v_scale.clone(), kvq.k_tail[:, :, :n].clone(), kvq.v_tail[:, :, :n].clone()))
    for a in got:
        for c in got:
            if a[0] == c[0]:
                assert all(torch.equal(x, y) for x, y in zip(a[1:], c[1:]))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_kvq_append_of_extreme_pages(fmt):
    """Zeros, the tiniest and the largest magnitudes, an infinity and a NaN."""
    table = torch.arange(8, dtype=torch.int32, device=DEV)[None]
    kvq = new_kvq_cache(8, 1, 1, 16, table, torch.tensor([96], dtype=torch.int32, device=DEV), fmt=fmt)
    ctx = context(1, 1, batch=1, pages=8)
    x = torch.randn(96, 1, 128, generator=torch.Generator().manual_seed(0))
    x[0:16] = 0
    x[16:32] *= 2.0 ** -110
    x[32:48] *= 2.0 ** 110
    x[48:64] *= 2.0 ** -90
    x[64, 0, 5] = float("inf")
    x[95, 0, 127] = float("nan")
    x = x.to(torch.bfloat16).to(DEV)
    ctx.locks_kvq_append(x, x, kvq, 1, cu_tokens=torch.tensor([0, 96], dtype=torch.int32, device=DEV))
    for name in ("k", "v"):
        for p in range(4):
            check_page(kvq, name, p, 0, U.f64(x[16 * p:16 * p + 16, 0]), fmt, torch.zeros(16, 128, dtype=torch.float64), (name, p))
        s = getattr(kvq, name + "_scale")[:, 0]
        assert bool(torch.isnan(s[4:6]).all()) and not bool(getattr(kvq, name)[4:6].float().any())


def test_kvq_append_skips_what_is_not_there():
    ctx = context(2, 1, batch=3, pages=2)
    gen = torch.Generator().manual_seed(3)
    k, v = rows(gen, 40, 1, "bf16"), rows(gen, 40, 1, "bf16")
    table = torch.tensor([[0, 1], [2, 1 << 30], [3, -1]], dtype=torch.int32, device=DEV)

    def run(lens, cu):
        kvq = new_kvq_cache(4, 3, 1, 16, table, torch.tensor(lens, dtype=torch.int32, device=DEV))
        ctx.locks_kvq_append(k, v, kvq, 3, cu_tokens=torch.tensor(cu, dtype=torch.int32, device=DEV))
        return ctx.locks_poll_status(), list(kvq.k_scale[:, 0].cpu() > 0), list(kvq.k_tail.abs().sum((1, 2, 3)).cpu() > 0)

    assert run([16, 8, 0], [0, 16, 24, 24]) == (0, [True, False, False, False], [False, True, False])
    # request 1: its second page has no block
    assert run([16, 32, 16], [0, 16, 32, 40]) == (-6, [True, False, False, True], [False, False, False])
    assert run([16, 32, 4], [0, 16, 36, 40]) == (-6, [True, False, True, False], [False, False, True])
    assert run([2 ** 31 - 1, 4, 4], [0, 1, 5, 9])[0] == -6
    st, pages, tails = run([8, 8, 8], [0, 9, 17, 25])              # request 0: more new tokens than it has
    assert st == -6 and tails == [False, True, True]
    st, pages, tails = run([20, 20, 20], [0, 20, 30, 50])          # request 2: rows that are not there
    assert st == -6 and pages[0] and tails == [True, True, False]
    st, pages, tails = run([40, 8, 8], [0, 40, 40, 40])            # 40 tokens in a row of 32
    assert st == -6 and pages[0] and pages[1] and tails == [False, False, False]


# ------------------------------------------------------------------------------------------------ attention
def run_attend(Hq, Hkv, B, fmt, layout, lens, new, pad=0, ids=None, cnt=None, budget=None, spread=0.0, seed=0, q_scale=2.0, change=None, **kw):
    batch, n = len(lens), sum(new) + pad
    gen = torch.Generator().manual_seed(seed + sum(lens))
    kvq = U.random_cache(gen, batch, lens, Hkv, B, fmt, layout, spread=spread)
    if change:
        change(kvq)
    ctx = context(Hq, Hkv, B=B, batch=batch + 1, pages=kvq.block_table.shape[1], budget=budget or 2 * B, **kw)
    q = (q_scale * torch.randn(n, Hq, 128, generator=gen)).to(torch.bfloat16).to(DEV)
    out = torch.full_like(q, 7.0)
    lse = torch.full((n, Hq), 7.0, device=DEV)
    many = pad or any(m != 1 for m in new)
    ctx.locks_kvq_attend(q, kvq, batch, out, lse, page_ids=ids, page_count=cnt, cu_tokens=U.cu_of(new, DEV) if many else None)
    return ctx, kvq, q, out, lse


def check_attend(Hq, Hkv, B, lens, new, kvq, q, out, lse, ids=None, cnt=None, per_head=False):
    live = sum(new)
    wo, wl, bo, bl = U.attend(q[:live], kvq, lens, new, Hkv, B, ids, cnt, per_head)
    near(out[:live], wo, bo, "out")
    got = U.f64(lse[:live])
    dead = torch.isinf(wl)
    assert torch.equal(got[dead], wl[dead])
    near(got[~dead], wl[~dead], bl[~dead], "lse")
    assert bool((out[live:] == 7.0).all()) and bool((lse[live:] == 7.0).all()), "rows behind the last request"


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("B,layout", [(16, "HND"), (16, "NHD"), (32, "NHD"), (64, "HND")])
@pytest.mark.parametrize("Hq,Hkv,lens", [(4, 1, [1]), (32, 8, [15, 16, 17, 0, 333]), (28, 4, [640]), (16, 1, [2000, 1, 64]), (10, 2, [31, 65]), (3, 3, [129, 48])])
def test_attend_one_token(Hq, Hkv, lens, B, layout, fmt):
    new = [1] * len(lens)
    ctx, kvq, q, out, lse = run_attend(Hq, Hkv, B, fmt, layout, lens, new)
    check_attend(Hq, Hkv, B, lens, new, kvq, q, out, lse)
    assert ctx.locks_poll_status() == 0


@pytest.mark.parametrize("B", [16, 32, 64])
@pytest.mark.parametrize("Hq,Hkv,lens,new,pad", [
    (8, 2, [33, 5, 200], [2, 5, 1], 0), (32, 8, [64, 100], [8, 3], 2), (16, 1, [70, 40, 9], [1, 0, 9], 1), (6, 2, [50], [50], 0),
    (7, 1, [37, 16], [5, 16], 0), (5, 1, [80, 96, 3], [17, 1, 3], 4)])
def test_attend_several_tokens(Hq, Hkv, lens, new, pad, B):
    ctx, kvq, q, out, lse = run_attend(Hq, Hkv, B, "int8" if B == 16 else "e4m3", "HND", lens, new, pad)
    check_attend(Hq, Hkv, B, lens, new, kvq, q, out, lse)
    assert ctx.locks_poll_status() == 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("B,layout", [(16, "HND"), (32, "NHD"), (64, "HND")])
@pytest.mark.parametrize("Hq,Hkv,lens,new,pad", [
    (64, 16, [130, 45, 300], [100, 45, 200], 3), (128, 16, [90, 64, 33], [90, 60, 1], 0), (176, 16, [200, 20], [140, 0], 1), (256, 16, [16, 81, 70], [16, 1, 64], 0),
    (20, 20, [1000], [1000], 2)])
def test_attend_chunks(Hq, Hkv, lens, new, pad, B, layout, fmt):
    """Enough rows per KV head for the form with 128 rows a tile."""
    ctx, kvq, q, out, lse = run_attend(Hq, Hkv, B, fmt, layout, lens, new, pad)
    check_attend(Hq, Hkv, B, lens, new, kvq, q, out, lse)
    assert ctx.locks_poll_status() == 0


def test_attend_long_sequences():
    """Shares of hundreds of tiles, in both forms of the token kernel, against torch in 64 bits on the GPU."""
    for Hq, Hkv, lens in ((32, 8, [300_000]), (32, 2, [700_000, 40_001]), (8, 8, [120_001, 7, 90_000, 33])):
        ctx, kvq, q, out, lse = run_attend(Hq, Hkv, 16, "int8", "HND", lens, [1] * len(lens))
        for b, t in enumerate(lens):
            for h in range(0, Hkv, max(1, Hkv // 2)):
                blocks = kvq.block_table[b, :t // 16].long()
                k, v = [torch.cat([(getattr(kvq, n)[blocks, h].double() * getattr(kvq, n + "_scale")[blocks, h].double()[:, None, None]).flatten(0, 1),
                                   getattr(kvq, n + "_tail")[b, h, :t % 16].double()]) for n in ("k", "v")]
                g = slice(h * Hq // Hkv, (h + 1) * Hq // Hkv)
                s = q[b, g].double() @ k.T * 128 ** -0.5
                want, ll = torch.softmax(s, 1) @ v, torch.logsumexp(s, 1)
                # 2^-8 of the result, 2^-11 of each weight; scores within 2^-16 of their magnitudes, which are below 200
                tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 200 * 2.0 ** -16) * 1.1 * (torch.softmax(s, 1) @ v.abs()) + 1e-4
                assert float(((out[b, g].double() - want).abs() - tol).max()) <= 0
                assert float((lse[b, g].double() - ll).abs().max()) <= 200 * 2.0 ** -16
        assert ctx.locks_poll_status() == 0


@pytest.mark.parametrize("B,combine", [(16, 0), (32, 0), (64, 0), (16, locks.COMBINE_PER_HEAD)])
def test_attend_listed_pages(B, combine):
    Hq, Hkv, lens, k = 8, 2, [16 * 40 + 3, 64, 30, 500, 0], 6
    per_head = combine == locks.COMBINE_PER_HEAD
    heads = Hq if per_head else Hkv
    gen = torch.Generator().manual_seed(B)
    ids, cnt = torch.full((5, heads, k), -1, dtype=torch.int32), torch.zeros(5, heads, dtype=torch.int32)
    for b, t in enumerate(lens):
        pages = -(-t // B)
        for h in range(heads):
            m = min(k, pages) if (b, h) != (1, 0) else 0   # one empty list
            cnt[b, h] = m
            ids[b, h, :m] = torch.randperm(pages, generator=gen)[:m].sort().values.to(torch.int32)
            if m and b == 0:
                ids[b, h, m - 1] = pages - 1
    new = [1] * 5
    ctx, kvq, q, out, lse = run_attend(Hq, Hkv, B, "int8", "HND", lens, new, ids=ids.to(DEV), cnt=cnt.to(DEV), budget=k * B, combine=combine)
    check_attend(Hq, Hkv, B, lens, new, kvq, q, out, lse, ids, cnt, per_head)
    assert ctx.locks_poll_status() == 0


def test_attend_scales_of_any_size():
    """Page scales over fourteen decades: no product of codes meets them."""
    lens = [700, 90]
    ctx, kvq, q, out, lse = run_attend(8, 2, 16, "int8", "HND", lens, [1, 1], spread=4.0, q_scale=0.01)
    check_attend(8, 2, 16, lens, [1, 1], kvq, q, out, lse)


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** 30])
def test_attend_queries_of_any_size(scale):
    lens = [300, 47]

    def change(kvq):   # keys such that the logits are ordinary
        kvq.k_scale.mul_(1 / scale)
        kvq.k_tail.mul_(1 / scale)
    ctx, kvq, q, out, lse = run_attend(8, 2, 16, "e4m3", "HND", lens, [1, 1], q_scale=2.0 * scale, change=change)
    check_attend(8, 2, 16, lens, [1, 1], kvq, q, out, lse)


@pytest.mark.parametrize("Hq,Hkv,n0", [(8, 2, 20), (64, 16, 300)])
def test_attend_infinities_and_nan(Hq, Hkv, n0):
    """Stale rows behind the last token are not looked at; a poisoned page makes NaN of what attends it and of nothing else; an
    infinite value in the unfinished page stays infinite, for the tokens that see it."""
    G = Hq // Hkv
    lens, new = ([37, 49], [3, 1]) if n0 == 20 else ([325, 49], [310, 30])

    def stale(kvq):
        for n in ("k_tail", "v_tail"):
            getattr(kvq, n)[0, :, 5:] = float("nan")
            getattr(kvq, n)[1, :, 1:] = float("inf")
        used = set(kvq.block_table[0, :lens[0] // 16].tolist() + kvq.block_table[1, :lens[1] // 16].tolist())
        for i in range(kvq.k.shape[0]):
            if i not in used:
                kvq.k_scale[i] = kvq.v_scale[i] = float("nan")
    ctx, kvq, q, out, lse = run_attend(Hq, Hkv, 16, "int8", "HND", lens, new, change=stale)
    check_attend(Hq, Hkv, 16, lens, new, kvq, q, out, lse)

    for which in ("k_scale", "v_scale"):
        def poison(kvq):
            getattr(kvq, which)[int(kvq.block_table[0, 1]), 0] = float("nan")   # places 16 .. 31, head 0
        T = n0 + 14   # the new tokens' places are 14 ..
        ctx, kvq, q, out, lse = run_attend(Hq, Hkv, 16, "int8", "HND", [T, 40], [n0, 1], change=poison)
        assert bool(torch.isnan(out[2:n0, :G]).all()), which
        fine = out.clone()
        fine[2:n0, :G] = 0
        assert not bool(torch.isnan(fine).any()), which

    def infinite(kvq):
        kvq.v_tail[0, 1, 2, 9] = float("inf")     # the third place of the unfinished page of request 0
    T, n = (37, 4) if n0 == 20 else (325, 310)
    ctx, kvq, q, out, lse = run_attend(Hq, Hkv, 16, "e4m3", "HND", [T, 40], [n, 1], change=infinite, q_scale=0.1)
    hit = torch.isinf(out)
    want = torch.zeros_like(hit)
    want[n - (T - T // 16 * 16 - 2):n, G:2 * G, 9] = True
    assert torch.equal(hit, want) and not bool(torch.isnan(out).any())


def test_attend_reports_bad_blocks_lengths_and_counts():
    lens = [100, 60]

    def bad(kvq):
        kvq.block_table[0, 2] = 1 << 29
        kvq.block_table[1, 1] = -4
    ctx, kvq, q, out, lse = run_attend(4, 2, 16, "int8", "HND", lens, [1, 1], change=bad)
    assert ctx.locks_poll_status() == -6 and not bool(torch.isnan(out).any())
    good = U.random_cache(torch.Generator().manual_seed(1), 2, lens, 2, 16, "int8")
    ctx = context(4, 2, batch=2, pages=good.block_table.shape[1])
    q, out = torch.randn(2, 4, 128, device=DEV).to(torch.bfloat16), torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=DEV)
    good.block_table.clamp_(max=3)
    for length in (-7, 16 * good.block_table.shape[1] + 1, 2 ** 31 - 1):
        good.seq_lens[1] = length
        ctx.locks_kvq_attend(q, good, 2, out)
        assert ctx.locks_poll_status() == (0 if length < 0 else -6)
        assert not bool(torch.isnan(out).any())
    good.seq_lens[1] = 60
    ids = torch.tensor([[[0, 1, -1, 5]] * 2, [[0, 3, 99, 2]] * 2], dtype=torch.int32, device=DEV)
    ctx = context(4, 2, batch=2, pages=good.block_table.shape[1], budget=64)
    ctx.locks_kvq_attend(q, good, 2, out, page_ids=ids, page_count=torch.tensor([[2, 9], [4, -1]], dtype=torch.int32, device=DEV))
    assert ctx.locks_poll_status() == -6
    ctx.locks_kvq_attend(q, good, 2, out, cu_tokens=torch.tensor([0, 1, 5], dtype=torch.int32, device=DEV))   # rows that are not there
    assert ctx.locks_poll_status() == -6


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("fmt,B,rank_fmt", [("int8", 16, "i4"), ("e4m3", 16, "bf16"), ("int8", 32, "i4")])
def test_a_prompt_and_decode_steps(fmt, B, rank_fmt):
    """Prompt in two chunks, summaries from the codes, then steps: append, select, attend, summaries of pages that filled."""
    Hq, Hkv, batch, budget = 8, 2, 2, 6 * B
    lens = [23 * B + 5, 9 * B + 15]
    gen = torch.Generator().manual_seed(5)
    Pmax = 28
    table = torch.randperm(batch * Pmax, generator=gen).to(torch.int32).view(batch, Pmax).to(DEV)
    ctx = locks.Context(make_config(Hq, Hkv, 8, rank_fmt, "bf16", batch, Pmax, budget, B=B), device=DEV)
    kvq = new_kvq_cache(batch * Pmax, batch, Hkv, B, table, torch.zeros(batch, dtype=torch.int32, device=DEV), fmt=fmt)
    rot = make_rotary(freqs(128))
    summ = ctx.new_summaries(batch * Pmax)
    done = [0, 0]
    for part in (0.4, 1.0):
        upto = [int(part * t) for t in lens]
        new = [u - d for u, d in zip(upto, done)]
        n = sum(new)
        kvq.seq_lens.copy_(torch.tensor(upto, dtype=torch.int32))
        q, k, v = rows(gen, n, Hq, "bf16"), rows(gen, n, Hkv, "bf16"), rows(gen, n, Hkv, "bf16")
        ctx.locks_kvq_append(k, v, kvq, batch, rotary=rot, q=q, q_out=q, cu_tokens=U.cu_of(new, DEV))
        out = torch.empty_like(q)
        lse = torch.empty(n, Hq, device=DEV)
        ctx.locks_kvq_attend(q, kvq, batch, out, lse, cu_tokens=U.cu_of(new, DEV))
        check_attend(Hq, Hkv, B, upto, new, kvq, q, out, lse)
        done = upto
    ctx.locks_kvq_build_summaries(kvq, batch, summ)
    k_ids = ctx.k
    ids = torch.empty(batch, Hkv, k_ids, dtype=torch.int32, device=DEV)
    cnt = torch.empty(batch, Hkv, dtype=torch.int32, device=DEV)
    for step in range(3):
        kvq.seq_lens += 1
        lens = [t + 1 for t in lens]
        q, k, v = rows(gen, batch, Hq, "bf16"), rows(gen, batch, Hkv, "bf16"), rows(gen, batch, Hkv, "bf16")
        ctx.locks_kvq_append(k, v, kvq, batch, rotary=rot, q=q, q_out=q)
        ctx.locks_select(q, summ, kvq.kv_view(), batch, ids, cnt)
        out, lse = torch.empty_like(q), torch.empty(batch, Hq, device=DEV)
        ctx.locks_kvq_attend(q, kvq, batch, out, lse, page_ids=ids, page_count=cnt)
        check_attend(Hq, Hkv, B, lens, [1, 1], kvq, q, out, lse, ids.cpu(), cnt.cpu())
        for b, t in enumerate(lens):   # the sink and the newest page are always there
            got = ids[b, 0, :int(cnt[b, 0])].tolist()
            assert got[0] == 0 and got[-1] == -(-t // B) - 1 and len(got) == min(-(-t // B), k_ids)
        full = torch.tensor([t // B for t in lens], dtype=torch.int32, device=DEV)
        first = torch.tensor([(t - 1) // B for t in lens], dtype=torch.int32, device=DEV)
        ctx.locks_kvq_build_summaries(kvq, batch, summ, first, full)
    assert ctx.locks_poll_status() == 0
    # the summaries are those of the values that the codes stand for: byte for byte what the builder makes of an fp32 cache that holds them
    real = kvq.k.float() * kvq.k_scale[:, :, None, None]
    ctx32 = locks.Context(make_config(Hq, Hkv, 8, rank_fmt, "f32", batch, Pmax, budget, B=B), device=DEV)
    want = ctx32.new_summaries(batch * Pmax)
    ctx32.locks_build_summaries(KVView(real, real, real.stride()[:3], batch * Pmax, table, kvq.seq_lens), batch, want)
    for b, t in enumerate(lens):
        blocks = table[b, :t // B].long()
        assert torch.equal(summ[blocks], want[blocks]) and bool((want[blocks] != 0).any(-1).all())


def test_two_streams_and_a_captured_step():
    """A captured append and attention replayed with other lengths and rows, on a stream of their own; and calls on two contexts at once."""
    Hq, Hkv, B, batch = 8, 2, 16, 3
    gen = torch.Generator().manual_seed(9)
    lens = [50, 31, 200]
    kvq = U.random_cache(gen, batch, [t + 40 for t in lens], Hkv, B, "int8")
    kvq.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    ctx = context(Hq, Hkv, B=B, batch=batch, pages=kvq.block_table.shape[1], budget=2 * B)
    rot = make_rotary(freqs(128))
    q, k, v = rows(gen, batch, Hq, "bf16"), rows(gen, batch, Hkv, "bf16"), rows(gen, batch, Hkv, "bf16")
    qo, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(batch, Hq, device=DEV)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()

    def step():
        ctx.locks_kvq_append(k, v, kvq, batch, rotary=rot, q=q, q_out=qo)
        ctx.locks_kvq_attend(qo, kvq, batch, out, lse)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kvq.seq_lens += 1
        step()
        with torch.cuda.graph(graph, stream=side):
            step()
        for i in range(20):
            kvq.seq_lens += 1
            q.copy_(rows(gen, batch, Hq, "bf16"))
            k.copy_(rows(gen, batch, Hkv, "bf16"))
            graph.replay()
            side.synchronize()
            now = [t + 2 + i for t in lens]
            check_attend(Hq, Hkv, B, now, [1] * batch, kvq, qo, out, lse)
    torch.cuda.current_stream().wait_stream(side)
    # two contexts, two streams, at once: the same results as one after the other
    ctx2 = context(Hq, Hkv, B=B, batch=batch, pages=kvq.block_table.shape[1], budget=2 * B)
    outs = [torch.empty_like(q) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for c, o, s in zip((ctx, ctx2), outs, streams):
            c.locks_kvq_attend(qo, kvq, batch, o, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], out) and torch.equal(outs[1], out)


def test_refusals():
    ctx = context(4, 2, batch=2, pages=4)
    kvq = new_kvq_cache(4, 2, 2, 16, torch.zeros(2, 4, dtype=torch.int32, device=DEV), torch.ones(2, dtype=torch.int32, device=DEV))
    q, out = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=DEV)
    k = torch.zeros(2, 2, 128, dtype=torch.bfloat16, device=DEV)
    rot = make_rotary(freqs(128))
    pos = torch.zeros(2, dtype=torch.int32, device=DEV)
    bad = [
        lambda: ctx.locks_rope(rot, pos, q.float(), out), lambda: ctx.locks_rope(rot, pos, q[:1], out), lambda: ctx.locks_rope(rot, pos.cpu(), q, out),
        lambda: ctx.locks_rope(rot, pos.long(), q, out), lambda: ctx.locks_rope(rot, pos, q, None), lambda: ctx.locks_rope(rot, None, q, out),
        lambda: ctx.locks_rope(rot, torch.zeros(3, 2, dtype=torch.int32, device=DEV), q, out), lambda: ctx.locks_rope(rot, pos, q.cpu(), out),
        lambda: ctx.locks_rope(rot, pos, q, torch.zeros(2, 4, 129, dtype=torch.bfloat16, device=DEV)[..., 1:]),
        lambda: ctx.locks_kvq_append(k, k[:1], kvq, 2), lambda: ctx.locks_kvq_append(k[:1], k[:1], kvq, 2), lambda: ctx.locks_kvq_append(k, k, kvq, 3),
        lambda: ctx.locks_kvq_append(k, k, kvq, 2, q=q, q_out=out), lambda: ctx.locks_kvq_append(k, k, kvq, 2, cu_tokens=pos),
        lambda: ctx.locks_kvq_attend(q, kvq, 2, out[:1]), lambda: ctx.locks_kvq_attend(q[:1], kvq, 2, out[:1]),
        lambda: ctx.locks_kvq_attend(q, kvq, 2, out, page_ids=torch.zeros(2, 2, 4, dtype=torch.int32, device=DEV)),
        lambda: ctx.locks_kvq_attend(q, kvq, 2, out, page_ids=torch.zeros(2, 2, 4, dtype=torch.int32, device=DEV), page_count=torch.zeros(2, 2, dtype=torch.int32, device=DEV),
                                     cu_tokens=torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)),
        lambda: context(4, 2, batch=2, pages=4, dtype="f32").locks_kvq_append(k.float(), k.float(), kvq, 2),
        lambda: context(8, 2, batch=2, pages=4).locks_kvq_attend(q, kvq, 2, out),
        lambda: context(4, 2, batch=2, pages=5).locks_kvq_attend(q, kvq, 2, out),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(locks.LocksError):
            f()
            print("not refused:", i)
    assert ctx.locks_poll_status() == 0


# ------------------------------------------------------------------------------------------------ chunks: shares, heads, scales
@pytest.mark.parametrize("fmt,B,layout", [("int8", 16, "HND"), ("e4m3", 32, "NHD"), ("int8", 64, "HND")])
@pytest.mark.parametrize("Hq,Hkv,lens,new,pad", [
    (32, 8, [32], [32], 0),                      # a share per tile, and more shares than tiles
    (32, 8, [2500], [40], 3),
    (32, 2, [1201, 700], [25, 24], 0),           # 16 heads a group, a second half of a block with one token
    (32, 2, [129], [129], 0),
    (8, 8, [640, 1000], [300, 129], 0),          # one head a group
    (15, 3, [400, 33, 0, 77], [90, 33, 0, 70], 9),
    (16, 1, [3001], [64], 200),
    (32, 8, [100 + 7 * i for i in range(40)], [30 + i % 3 for i in range(40)], 0)])
def test_attend_chunks_in_shares(Hq, Hkv, lens, new, pad, fmt, B, layout):
    """Few blocks of rows, so that several CTAs share the tokens of each; more requests than a warp has lanes."""
    ctx, kvq, q, out, lse = run_attend(Hq, Hkv, B, fmt, layout, lens, new, pad)
    check_attend(Hq, Hkv, B, lens, new, kvq, q, out, lse)
    assert ctx.locks_poll_status() == 0


@pytest.mark.parametrize("Hkv", [1, 16])
def test_attend_chunks_take_nothing_of_later_pages(Hkv):
    """Later pages of the chunk hold far larger values: rows that do not see them lose nothing to them."""
    lens, new = [256], [256]

    def change(kvq):
        for p in range(16):
            kvq.v_scale[kvq.block_table[0, p].long()] *= 2.0 ** (3 * p)

    ctx, kvq, q, out, lse = run_attend(4 * Hkv, Hkv, 16, "int8", "HND", lens, new, change=change)
    check_attend(4 * Hkv, Hkv, 16, lens, new, kvq, q, out, lse)


def test_attend_chunks_scales_of_any_size():
    lens, new = [700, 190], [100, 60]
    ctx, kvq, q, out, lse = run_attend(8, 2, 16, "int8", "HND", lens, new, spread=4.0, q_scale=0.01)
    check_attend(8, 2, 16, lens, new, kvq, q, out, lse)


@pytest.mark.parametrize("Hq,Hkv,T,m", [(32, 8, 100_003, 32), (16, 1, 50_016, 90)])
def test_attend_chunks_of_long_sequences(Hq, Hkv, T, m):
    """Hundreds of tiles a share, against torch in 64 bits on the GPU."""
    ctx, kvq, q, out, lse = run_attend(Hq, Hkv, 16, "e4m3", "HND", [T], [m])
    G, blocks = Hq // Hkv, kvq.block_table[0, :T // 16].long()
    see = torch.arange(T, device=DEV)[None] < (T - m + 1 + torch.arange(m, device=DEV))[:, None]
    for h in {0, Hkv - 1}:
        k, v = [torch.cat([(getattr(kvq, n)[blocks, h].double() * getattr(kvq, n + "_scale")[blocks, h].double()[:, None, None]).flatten(0, 1),
                           getattr(kvq, n + "_tail")[0, h, :T % 16].double()]) for n in ("k", "v")]
        s = torch.einsum("mgd,td->mgt", q[:, h * G:h * G + G].double(), k) * 128 ** -0.5
        s = s.masked_fill(~see[:, None], -math.inf)
        p = torch.softmax(s, 2)
        want, ll = p @ v, torch.logsumexp(s, 2)
        # 2^-8 of the result, 2^-11 of each weight; scores within 2^-16 of their magnitudes, which are below 200
        tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 200 * 2.0 ** -16) * 1.1 * (p @ v.abs()) + 1e-4
        assert float(((out[:, h * G:h * G + G].double() - want).abs() - tol).max()) <= 0
        assert float((lse[:, h * G:h * G + G].double() - ll).abs().max()) <= 200 * 2.0 ** -16
    assert ctx.locks_poll_status() == 0


def test_attend_chunks_infinities_and_nan():
    """An infinite value and a NaN key in the unfinished page reach the rows that see them, and no other; a page whose scale is NaN too."""
    Hq, Hkv, T, m = 16, 4, 203, 60

    def change(kvq):
        kvq.v_tail[0, 1, 3, 7] = float("inf")
        kvq.k_tail[0, 2, 5, 9] = float("nan")
        kvq.k_scale[int(kvq.block_table[0, 11]), 3] = float("nan")

    ctx, kvq, q, out, lse = run_attend(Hq, Hkv, 16, "int8", "HND", [T], [m], change=change)
    o, l = out.float(), lse
    first = T - m                      # row j sees tokens 0 .. first + j
    tail, page = T // 16 * 16, 11 * 16
    for j in range(m):
        g = lambda h: slice(4 * h, 4 * h + 4)
        assert bool(torch.isfinite(o[j, g(0)]).all())
        assert bool((o[j, g(1), 7] == float("inf")).all()) == (first + j >= tail + 3)
        assert bool(torch.isfinite(o[j, g(1), :7]).all() and torch.isfinite(o[j, g(1), 8:]).all() and torch.isfinite(l[j, g(1)]).all())
        assert bool(torch.isnan(o[j, g(2)]).all()) == (first + j >= tail + 5) and bool(torch.isfinite(o[j, g(2)]).all()) == (first + j < tail + 5)
        assert bool(torch.isnan(o[j, g(3)]).all()) == (first + j >= page) and bool(torch.isfinite(o[j, g(3)]).all()) == (first + j < page)
    assert ctx.locks_poll_status() == 0


def test_attend_chunks_report_bad_blocks_and_rows():
    Hq, Hkv = 32, 8
    ctx, kvq, q, out, lse = run_attend(Hq, Hkv, 16, "int8", "HND", [200, 90], [40, 40])
    assert ctx.locks_poll_status() == 0
    # rows that are not there, and a request before them: its rows are answered, those of the other not
    out.fill_(7.0)
    ctx.locks_kvq_attend(q, kvq, 2, out, lse, cu_tokens=torch.tensor([0, 40, 100], dtype=torch.int32, device=DEV))
    assert ctx.locks_poll_status() == -6
    check_attend(Hq, Hkv, 16, [200], [40], kvq, q[:40], out[:40], lse[:40])
    assert bool((out[40:] == 7.0).all())
    # a block outside the cache: none of its tokens are seen
    kvq.block_table[0, 0] = -3
    ctx.locks_kvq_attend(q, kvq, 2, out, lse, cu_tokens=U.cu_of([40, 40], DEV))
    assert ctx.locks_poll_status() == -6 and bool(torch.isfinite(out.float()).all())
    check_attend(Hq, Hkv, 16, [90], [40], _second(kvq), q[40:], out[40:], lse[40:])


def _second(kvq):
    """The cache as its second request sees it."""
    import copy
    one = copy.copy(kvq)
    one.block_table, one.seq_lens = kvq.block_table[1:], kvq.seq_lens[1:]
    one.k_tail, one.v_tail = kvq.k_tail[1:], kvq.v_tail[1:]
    return one


# ------------------------------------------------------------------------------------------------ many requests, far rows, repeated pages
@pytest.mark.parametrize("Hq,Hkv,some", [(8, 2, False), (8, 2, True), (16, 1, True)])
def test_attend_more_requests_than_lanes(Hq, Hkv, some):
    lens = [(37 * i) % 150 for i in range(75)]
    new = [min(t, 1 + (i % 3 if some else 0)) for i, t in enumerate(lens)]
    if not some:
        new = [1] * 75
    ctx, kvq, q, out, lse = run_attend(Hq, Hkv, 16, "int8", "HND", lens, new, 2 if some else 0)
    check_attend(Hq, Hkv, 16, lens, new, kvq, q, out, lse)
    assert ctx.locks_poll_status() == 0


def test_attend_a_page_listed_twice_counts_twice():
    lens, k, B = [16 * 20 + 5], 6, 16
    ids = torch.tensor([[[3, 3, 7, 20, 20, 2], [20, 20, 20, 1, 1, 1]]], dtype=torch.int32)
    cnt = torch.tensor([[6, 4]], dtype=torch.int32)
    ctx, kvq, q, out, lse = run_attend(8, 2, B, "int8", "HND", lens, [1], ids=ids.to(DEV), cnt=cnt.to(DEV), budget=k * B)
    check_attend(8, 2, B, lens, [1], kvq, q, out, lse, ids, cnt)
    assert ctx.locks_poll_status() == 0


@pytest.mark.parametrize("n", [1, 40])
def test_attend_and_append_far_into_a_large_cache(n):
    """Blocks beyond 2^32 bytes, and strides that are not the tensors' own order."""
    Hq, Hkv, B, T, stride = 32, 8, 16, 100, 1 << 26
    gen = torch.Generator().manual_seed(n)
    small = U.random_cache(gen, 1, [T], Hkv, B, "int8")
    nb = 68
    big = [torch.empty((nb - 1) * stride + Hkv * B * 128, dtype=torch.int8, device=DEV) for _ in range(2)]
    k, v = [t.as_strided((nb, Hkv, B, 128), (stride, B * 128, 128, 1)) for t in big]
    table = small.block_table.clone()
    ks, vs = torch.zeros(nb, Hkv, device=DEV), torch.zeros(nb, Hkv, device=DEV)
    for p in range(T // B):
        old, at = int(table[0, p]), nb - 1 - p
        k[at], v[at], ks[at], vs[at] = small.k[old], small.v[old], small.k_scale[old], small.v_scale[old]
        table[0, p] = at
    table[0, T // B] = nb - 1 - T // B
    kvq = locks.KVQView(k, v, ks, vs, small.k_tail, small.v_tail, table, small.seq_lens)
    ctx = context(Hq, Hkv, batch=2, pages=table.shape[1])
    # the page's last tokens, then attention of the last n
    x, y = rows(gen, 12, Hkv, "bf16"), rows(gen, 12, Hkv, "bf16")
    kvq.seq_lens.fill_(T + 12)
    ctx.locks_kvq_append(x, y, kvq, 1, cu_tokens=U.cu_of([12], DEV))
    q = torch.randn(n, Hq, 128, generator=gen).to(torch.bfloat16).to(DEV)
    out, lse = torch.empty_like(q), torch.empty(n, Hq, device=DEV)
    ctx.locks_kvq_attend(q, kvq, 1, out, lse, cu_tokens=U.cu_of([n], DEV))
    assert float(ks[nb - 1 - T // B].min()) > 0
    check_attend(Hq, Hkv, B, [T + 12], [n], kvq, q, out, lse)
    assert ctx.locks_poll_status() == 0


def test_appends_of_more_requests_than_threads():
    """300 requests: lookups that walk the requests in steps."""
    Hkv, B, batch = 2, 16, 300
    new = [(7 * i) % 4 for i in range(batch)]
    lens = [m + (5 * i) % 30 for i, m in enumerate(new)]
    n = sum(new)
    gen = torch.Generator().manual_seed(5)
    k, v = rows(gen, n, Hkv, "bf16"), rows(gen, n, Hkv, "bf16")
    pages = [-(-t // B) for t in lens]
    table = torch.full((batch, 3), -1, dtype=torch.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = torch.arange(at, at + p)
        at += p
    cu = U.cu_of(new, DEV)
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ctx = context(2, Hkv, B=B, batch=batch, pages=3)
    kc, vc = [torch.zeros(at, Hkv, B, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    kv = KVView(kc, vc, kc.stride()[:3], at, table.to(DEV), seq)
    ctx.locks_append_rows(k, v, kv, batch, cu_tokens=cu)
    kvq = new_kvq_cache(at, batch, Hkv, B, table.to(DEV), seq)
    ctx.locks_kvq_append(k, v, kvq, batch, cu_tokens=cu)
    assert ctx.locks_poll_status() == 0
    row = 0
    for b, (t, m) in enumerate(zip(lens, new)):
        for j in range(m):
            pos = t - m + j
            blk = int(table[b, pos // B])
            assert torch.equal(kc[blk, :, pos % B], k[row]) and torch.equal(vc[blk, :, pos % B], v[row])
            if pos >= t // B * B:
                assert torch.equal(kvq.k_tail[b, :, pos % B], k[row].float()) and torch.equal(kvq.v_tail[b, :, pos % B], v[row].float())
            row += 1
    assert row == n


def test_chunks_captured_on_streams_and_between_other_forms():
    """A captured chunk (append and attention, its tokens shared by several CTAs) replayed with other lengths; token and chunk forms in turn,
    which use one workspace; two contexts at once, bit for bit."""
    Hq, Hkv, B, m = 32, 8, 16, 40
    gen = torch.Generator().manual_seed(11)
    room, at = [700, 500], [120, 77]
    kvq = U.random_cache(gen, 2, room, Hkv, B, "e4m3")
    kvq.seq_lens.copy_(torch.tensor(at, dtype=torch.int32))
    for n in ("k", "v"):   # (the cache of a sequence of those lengths: its unfinished page in the tail)
        getattr(kvq, n + "_tail").copy_(torch.randn(2, Hkv, B, 128, generator=gen).to(DEV))
    ctx = context(Hq, Hkv, B=B, batch=2, pages=kvq.block_table.shape[1], budget=2 * B)
    rot = make_rotary(freqs(128))
    cu = U.cu_of([m, m], DEV)
    q, k, v = rows(gen, 2 * m, Hq, "bf16"), rows(gen, 2 * m, Hkv, "bf16"), rows(gen, 2 * m, Hkv, "bf16")
    qo, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(2 * m, Hq, device=DEV)
    one, one_lse = torch.empty(2, Hq, 128, dtype=torch.bfloat16, device=DEV), torch.empty(2, Hq, device=DEV)

    def step():
        ctx.locks_kvq_append(k, v, kvq, 2, rotary=rot, q=q, q_out=qo, cu_tokens=cu)
        ctx.locks_kvq_attend(qo, kvq, 2, out, lse, cu_tokens=cu)
        ctx.locks_kvq_attend(qo[:2], kvq, 2, one, one_lse)
        ctx.locks_kvq_attend(qo, kvq, 2, out, lse, cu_tokens=cu)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kvq.seq_lens += m
        step()
        with torch.cuda.graph(graph, stream=side):
            step()
        for i in range(6):
            kvq.seq_lens += m
            for t, h in ((q, Hq), (k, Hkv), (v, Hkv)):
                t.copy_(rows(gen, 2 * m, h, "bf16"))
            graph.replay()
            side.synchronize()
            now = [t + (2 + i) * m for t in at]
            check_attend(Hq, Hkv, B, now, [m, m], kvq, qo, out, lse)
            check_attend(Hq, Hkv, B, now, [1, 1], kvq, qo[:2], one, one_lse)
    torch.cuda.current_stream().wait_stream(side)
    ctx2 = context(Hq, Hkv, B=B, batch=2, pages=kvq.block_table.shape[1], budget=2 * B)
    outs, streams = [torch.empty_like(q) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for c, o, s in zip((ctx, ctx2), outs, streams):
            c.locks_kvq_attend(qo, kvq, 2, o, cu_tokens=cu, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], out) and torch.equal(outs[1], out)
    assert ctx.locks_poll_status() == 0 and ctx2.locks_poll_status() == 0


@pytest.mark.parametrize("new", [[1, 1], [3, 2]])
def test_attend_takes_no_unfinished_page_behind_the_table(new):
    """A length beyond an odd row of the table is reported; the pages that are there are attended, the unfinished one is not."""
    Hq, Hkv, B, pages = 8, 2, 16, 5
    lens = [pages * B + 7, 40]
    gen = torch.Generator().manual_seed(2)
    kvq = U.random_cache(gen, 2, lens, Hkv, B, "int8", rows_more=0)
    kvq.block_table = kvq.block_table[:, :pages].contiguous()
    ctx = context(Hq, Hkv, B=B, batch=2, pages=pages, budget=2 * B)
    n = sum(new)
    q = torch.randn(n, Hq, 128, generator=gen).to(torch.bfloat16).to(DEV)
    out, lse = torch.empty_like(q), torch.empty(n, Hq, device=DEV)
    ctx.locks_kvq_attend(q, kvq, 2, out, lse, cu_tokens=U.cu_of(new, DEV) if n > 2 else None)
    assert ctx.locks_poll_status() == -6
    # every row of the first request sees its 80 tokens in pages
    k, v, _ = U.sequence(kvq, 0, 0, pages * B, B)
    k1, v1, _ = U.sequence(kvq, 0, 1, pages * B, B)
    for h, (kk, vv) in enumerate(((k, v), (k1, v1))):
        s = U.f64(q[:new[0], 4 * h:4 * h + 4]) @ kk.T * 128 ** -0.5
        want, ll = torch.softmax(s, -1) @ vv, torch.logsumexp(s, -1)
        # 2^-8 of the result, 2^-11 of each weight; scores within 2^-16 of their magnitudes, which are below 100; 17 x 255 x 2^-23 of a scale (below 0.1)
        tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 100 * 2.0 ** -16) * 1.1 * (torch.softmax(s, -1) @ vv.abs()) + 17 * 255 * 2.0 ** -23 * 0.1
        near(out[:new[0], 4 * h:4 * h + 4], want, tol, "out")
        near(lse[:new[0], 4 * h:4 * h + 4], ll, torch.full_like(ll, 100 * 2.0 ** -16), "lse")
