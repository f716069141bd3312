"""GPU: the 8-bit cache's calls at offsets, lengths, elements and layouts that ordinary batches do not have."""
import math

import pytest
import torch

import kvq_util as U
import paper_2607_24555_b200 as locks
from paper_2607_24555_b200.binding import new_kvq_cache
from test_gpu_kvq import DEV, check_attend, context, near, rows

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ offsets
def test_attend_offsets_that_give_rows_to_many_requests():
    """Offsets that go up and down give every other request all rows: 400 tiles of rows each, of 65536 tokens, for 801 requests and 8 heads,
    are more work than 32 bits number.  Reported, and nothing is written."""
    batch, n, pages, heads = 1602, 24039, 4096, 8
    table = torch.zeros(batch, pages, dtype=torch.int32, device=DEV)
    kvq = new_kvq_cache(1, batch, heads, 16, table, torch.full((batch,), 16 * pages, dtype=torch.int32, device=DEV))
    ctx = context(heads, heads, batch=batch, pages=pages)
    q = torch.zeros(n, heads, 128, dtype=torch.bfloat16, device=DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((n, heads), 7.0, device=DEV)
    cu = torch.tensor([0 if b % 2 == 0 else n for b in range(batch + 1)], dtype=torch.int32, device=DEV)
    ctx.locks_kvq_attend(q, kvq, batch, out, lse, cu_tokens=cu)
    assert ctx.locks_poll_status() == -6
    assert bool((out == 7.0).all()) and bool((lse == 7.0).all())
    # and the context serves the next call
    lens = [40, 77]
    good = U.random_cache(torch.Generator().manual_seed(1), 2, lens, heads, 16, "int8", rows_more=pages - 5)
    q = torch.randn(5, heads, 128, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((5, heads), 7.0, device=DEV)
    ctx.locks_kvq_attend(q, good, 2, out, lse, cu_tokens=U.cu_of([2, 3], DEV))
    check_attend(heads, heads, 16, lens, [2, 3], good, q, out, lse)
    assert ctx.locks_poll_status() == 0


@pytest.mark.parametrize("Hq,Hkv,n", [(8, 2, 6), (64, 16, 300)])
def test_attend_offsets_that_go_back(Hq, Hkv, n):
    """A request whose offsets descend is reported and has no rows; those of the others are answered.  Both forms."""
    lens = [350, 40, 333]
    kvq = U.random_cache(torch.Generator().manual_seed(3), 3, lens, Hkv, 16, "int8")
    ctx = context(Hq, Hkv, batch=3, pages=kvq.block_table.shape[1], budget=128)
    q = torch.randn(2 * n, Hq, 128, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((2 * n, Hq), 7.0, device=DEV)
    cu = torch.tensor([0, n, n - 2, 2 * n - 2], dtype=torch.int32, device=DEV)
    ctx.locks_kvq_attend(q, kvq, 3, out, lse, cu_tokens=cu)
    assert ctx.locks_poll_status() == -6
    # rows that one request alone has; two rows are of two requests, and hold what either makes of them
    wo, _, bo, _ = U.attend(q[:n], kvq, lens[:1], [n], Hkv, 16)
    near(out[:n - 2], wo[:n - 2], bo[:n - 2], "first")
    last = _request(kvq, 2)
    wo, _, bo, _ = U.attend(q[n - 2:2 * n - 2], last, lens[2:], [n], Hkv, 16)
    near(out[n:2 * n - 2], wo[2:], bo[2:], "third")
    assert bool((out[2 * n - 2:] == 7.0).all())


def _request(kvq, b):
    import copy
    one = copy.copy(kvq)
    one.block_table, one.seq_lens = kvq.block_table[b:], kvq.seq_lens[b:]
    one.k_tail, one.v_tail = kvq.k_tail[b:], kvq.v_tail[b:]
    return one


# ------------------------------------------------------------------------------------------------ queries whose elements differ much in size
# What fp16 queries may move a score by: every element within 2^-25 of its row's largest, times the sum of a key's magnitudes.
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,new", [(8, 2, 1), (16, 1, 1), (8, 2, 3), (64, 16, 100)])
def test_attend_query_elements_below_the_largest(Hq, Hkv, new, fmt):
    """One large element that meets codes of zero, and 127 of 0.97 x 2^-25 of it: scores are the small ones' alone, the same to within their
    rounding whatever a page's scale is.  (Signed codes are multiplied as code + 128: what that adds has to be taken off as the products have it.)"""
    T, B, gen = 128, 16, torch.Generator().manual_seed(7)
    kvq = U.random_cache(gen, 1, [T], Hkv, B, fmt)
    codes = torch.randint(-1, 2, kvq.k.shape, generator=gen).float()
    codes[..., 0] = 0
    kvq.k.copy_(codes.to(kvq.k.dtype).to(DEV))
    kvq.k_scale.copy_((2.0 ** torch.randint(0, 3, kvq.k_scale.shape, generator=gen)).to(DEV))
    ctx = context(Hq, Hkv, B=B, batch=1, pages=kvq.block_table.shape[1], budget=128)
    q = torch.full((new, Hq, 128), 2.0 ** 16 * 0.96875 * 2.0 ** -25)
    q[..., 0] = 2.0 ** 16
    q = q.to(torch.bfloat16).to(DEV)
    out, lse = torch.empty_like(q), torch.empty(new, Hq, device=DEV)
    ctx.locks_kvq_attend(q, kvq, 1, out, lse, cu_tokens=U.cu_of([new], DEV))
    wo, wl, bo, bl = U.attend(q, kvq, [T], [new], Hkv, B)
    more = 2.0 ** -25 * 2.0 ** 16 * 127 * 4 * 128 ** -0.5   # (codes -1 .. 1, scales up to 4)
    assert more < 0.1
    vmax = max(float(U.sequence(kvq, 0, h, T, B)[1].abs().max()) for h in range(Hkv))
    near(out, wo, bo + 2 * math.expm1(more) * vmax, "out")
    near(lse, wl, bl + more, "lse")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,lens,new", [(8, 2, [300, 47], [1, 1]), (16, 1, [200], [2]), (64, 16, [210, 333], [90, 140])])
def test_attend_query_elements_of_all_sizes(Hq, Hkv, lens, new, fmt):
    """Elements of a row spread over 2^-30 .. 1."""
    gen = torch.Generator().manual_seed(8)
    kvq = U.random_cache(gen, len(lens), lens, Hkv, 16, fmt)
    ctx = context(Hq, Hkv, batch=len(lens), pages=kvq.block_table.shape[1], budget=128)
    n = sum(new)
    q = (4.0 * torch.randn(n, Hq, 128, generator=gen) * 2.0 ** (-30 * torch.rand(n, Hq, 128, generator=gen))).to(torch.bfloat16).to(DEV)
    out, lse = torch.empty_like(q), torch.empty(n, Hq, device=DEV)
    ctx.locks_kvq_attend(q, kvq, len(lens), out, lse, cu_tokens=U.cu_of(new, DEV))
    wo, wl, bo, bl = U.attend(q, kvq, lens, new, Hkv, 16)
    kmax = max(float(U.sequence(kvq, b, h, t, 16)[0].abs().sum(-1).max()) for b, t in enumerate(lens) for h in range(Hkv))
    vmax = max(float(U.sequence(kvq, b, h, t, 16)[1].abs().max()) for b, t in enumerate(lens) for h in range(Hkv))
    more = 2.0 ** -25 * float(U.f64(q).abs().max()) * kmax * 128 ** -0.5
    assert more < 1e-3
    near(out, wo, bo + 2 * math.expm1(more) * vmax, "out")
    near(lse, wl, bl + more, "lse")
    assert ctx.locks_poll_status() == 0


# ------------------------------------------------------------------------------------------------ long sequences, page by page
def marked_cache(gen, lens, Hkv, B, fmt, layout):
    """Every page has scales of its own; keys have a code of one in dimension 0 (which alone the queries have), values one in the
    dimension that the page's number gives.  So a page that is lost, taken twice or taken with another's scale shows."""
    batch, pages = len(lens), [-(-t // B) for t in lens]
    nb = sum(pages)
    order = torch.randperm(nb, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((batch, max(pages) + 1), 1 << 30, dtype=torch.int32, device=DEV)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = order[at:at + p]
        at += p
    kvq = new_kvq_cache(nb, batch, Hkv, B, table, torch.tensor(lens, dtype=torch.int32, device=DEV), fmt=fmt, layout=layout)
    for s, lo in ((kvq.k_scale, 0.5), (kvq.v_scale, 0.5)):
        s.copy_(lo * 4.0 ** torch.rand(s.shape, generator=gen, device=DEV))
    kvq.k[..., 0] = torch.ones(1, device=DEV).to(kvq.k.dtype)
    for b, p in enumerate(pages):
        v = torch.zeros(p, Hkv, B, 128, device=DEV)
        v[torch.arange(p, device=DEV), :, :, torch.arange(p, device=DEV) % 128] = 1.0
        kvq.v[table[b, :p].long()] = v.to(kvq.v.dtype)
        del v
        last = lens[b] // B
        kvq.k_tail[b, :, :, 0] = 0.75
        kvq.v_tail[b, :, :, last % 128] = 1.25
    return kvq


def marked_answer(kvq, b, h, T, B, a, pages, sees):
    """64 bits: (mean of values, log of the weights' sum) for queries a in dimension 0 over `pages` in that order, a row with `sees` tokens."""
    whole = T // B
    blocks = kvq.block_table[b, pages.clamp(max=whole)].long().clamp(0, kvq.k.shape[0] - 1)
    ks = torch.where(pages < whole, kvq.k_scale[blocks, h].double(), 0.75)
    vs = torch.where(pages < whole, kvq.v_scale[blocks, h].double(), 1.25)
    count = (sees - pages * B).clamp(0, B).double()
    w = torch.exp(a[:, None].double() * ks * 128 ** -0.5) * count
    total = w.sum(1)
    out = torch.zeros(len(a), 128, dtype=torch.float64, device=DEV).index_add_(1, pages % 128, w * vs) / total[:, None]
    return out, torch.log(total)


def check_marked(got, lse, want, ll, fmt, what):
    """A score is one product (exact) times a row's and a page's factor (|s| <= 0.5; four roundings: 2^-23), its exponential within 2^-22, and
    a sum is of at most 256 numbers one after the other, and as many partials (2^-15): 2^-14 in all; a page of 16 tokens among 10^5 is 2^-13 to 2^-12.
    Outputs are rounded (2^-8) as weights are (2^-11; with the value's scale, once more); signed codes: 17 x 255 x 2^-23 of a scale (up to 2)."""
    assert float((lse.double() - ll).abs().max()) <= 2.0 ** -14, what
    tol = want.abs() * (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -13) + (17 * 255 * 2.0 ** -23 * 2 if fmt == "int8" else 0.0) + 1e-6
    assert float(((got.double() - want).abs() - tol).max()) <= 0, what


def marked_queries(n, Hq):
    q = torch.zeros(n, Hq, 128, dtype=torch.bfloat16, device=DEV)
    q[..., 0] = (2.8 * (0.3 + 0.7 * torch.arange(Hq, device=DEV) / Hq) * (1 - 2 * (torch.arange(Hq, device=DEV) % 2))).to(torch.bfloat16)
    return q


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,B,layout,lens", [
    (32, 8, 16, "HND", [32_005, 31_000, 29_999, 32_768, 30_001, 8_200, 25_000, 16_384]),
    (32, 2, 16, "NHD", [60_003, 59_000, 61_111, 33, 64_000, 50_050, 60_000, 62_001, 40_000, 47_007]),
    (8, 2, 32, "NHD", [61_005, 60_000, 59_000, 44, 1, 60_032, 55_555, 32_768, 64_001, 63_000, 50_000, 61_000, 60_001, 60_002, 60_003, 50_001]),
    (8, 4, 64, "HND", [61_005, 60_000, 59_000, 60_032, 55_555, 32_768, 64_001, 30_000])])
def test_attend_every_page_of_long_sequences(Hq, Hkv, B, layout, lens, fmt):
    """Warps with many batches of blocks and scales: tens of pairs of tiles each."""
    gen = torch.Generator(device=DEV).manual_seed(sum(lens))
    kvq = marked_cache(gen, lens, Hkv, B, fmt, layout)
    batch, G = len(lens), Hq // Hkv
    ctx = context(Hq, Hkv, B=B, batch=batch, pages=kvq.block_table.shape[1], budget=128)
    q = marked_queries(batch, Hq)
    out, lse = torch.full_like(q, 7.0), torch.full((batch, Hq), 7.0, device=DEV)
    ctx.locks_kvq_attend(q, kvq, batch, out, lse)
    assert ctx.locks_poll_status() == 0
    for b, t in enumerate(lens):
        pages = torch.arange(-(-t // B), device=DEV)
        for h in range(Hkv):
            heads = slice(h * G, h * G + G)
            want, ll = marked_answer(kvq, b, h, t, B, q[b, heads, 0], pages, t)
            check_marked(out[b, heads], lse[b, heads], want, ll, fmt, (b, h))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("per_head", [False, True])
def test_attend_every_listed_page(fmt, per_head):
    """A thousand pages of each head in any order, the unfinished one among them."""
    Hq, Hkv, B, k, lens = 32, 8, 16, 1024, [40_005, 33_000, 20_000, 31_111, 16_390, 30_000, 28_001, 17_000]
    gen = torch.Generator(device=DEV).manual_seed(3)
    kvq = marked_cache(gen, lens, Hkv, B, fmt, "HND")
    batch, G, tables = len(lens), Hq // Hkv, Hq if per_head else Hkv
    more = {"combine": locks.COMBINE_PER_HEAD} if per_head else {}
    ctx = context(Hq, Hkv, B=B, batch=batch, pages=kvq.block_table.shape[1], budget=k * B, **more)
    ids = torch.zeros(batch, tables, k, dtype=torch.int32, device=DEV)
    cnt = torch.full((batch, tables), k, dtype=torch.int32, device=DEV)
    for b, t in enumerate(lens):
        pages = -(-t // B)
        for h in range(tables):
            ids[b, h] = torch.randperm(pages - 1, generator=gen, device=DEV)[:k].to(torch.int32)
            ids[b, h, (7 * h + b) % k] = pages - 1
            cnt[b, h] = k - (h * b) % 50
    q = marked_queries(batch, Hq)
    out, lse = torch.full_like(q, 7.0), torch.full((batch, Hq), 7.0, device=DEV)
    ctx.locks_kvq_attend(q, kvq, batch, out, lse, page_ids=ids, page_count=cnt)
    assert ctx.locks_poll_status() == 0
    for b, t in enumerate(lens):
        for i in range(tables):
            heads = slice(i, i + 1) if per_head else slice(i * G, i * G + G)
            pages = ids[b, i, :int(cnt[b, i])].long()
            want, ll = marked_answer(kvq, b, i // G if per_head else i, t, B, q[b, heads, 0], pages, t)
            check_marked(out[b, heads], lse[b, heads], want, ll, fmt, (b, i))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,B,lens,new", [(32, 8, 16, [100_003], [32]), (32, 8, 16, [40_000, 30_005], [300, 299]), (64, 16, 32, [50_001, 7_000, 22_222], [64, 64, 40]),
                                               (16, 1, 64, [90_016], [60]), (32, 8, 16, [50_005, 60_000], [3, 2])])
def test_chunks_attend_every_page_of_long_sequences(Hq, Hkv, B, lens, new, fmt):
    gen = torch.Generator(device=DEV).manual_seed(sum(lens))
    kvq = marked_cache(gen, lens, Hkv, B, fmt, "HND")
    batch, G, n = len(lens), Hq // Hkv, sum(new)
    ctx = context(Hq, Hkv, B=B, batch=batch, pages=kvq.block_table.shape[1], budget=128)
    q = marked_queries(n, Hq)
    out, lse = torch.full_like(q, 7.0), torch.full((n, Hq), 7.0, device=DEV)
    ctx.locks_kvq_attend(q, kvq, batch, out, lse, cu_tokens=U.cu_of(new, DEV))
    assert ctx.locks_poll_status() == 0
    row = 0
    for b, (t, m) in enumerate(zip(lens, new)):
        pages = torch.arange(-(-t // B), device=DEV)
        for j in {0, 1, m // 2, m - 1}:
            for h in {0, Hkv // 2, Hkv - 1}:
                heads = slice(h * G, h * G + G)
                want, ll = marked_answer(kvq, b, h, t, B, q[row + j, heads, 0], pages, t - m + j + 1)
                check_marked(out[row + j, heads], lse[row + j, heads], want, ll, fmt, (b, j, h))
        row += m


# ------------------------------------------------------------------------------------------------ lengths
@pytest.mark.parametrize("Hq,Hkv,new", [(8, 2, [1, 1, 1]), (8, 2, [3, 2, 4]), (64, 16, [100, 120, 90])])
@pytest.mark.parametrize("length", [0, -1, -7, -16, -2 ** 31])
def test_attend_empty_and_negative_lengths(Hq, Hkv, new, length):
    """A sequence with nothing in it: zeros and -inf, whatever is in its tail, and nothing of it in the others' rows."""
    lens = [200, 0, 133]
    kvq = U.random_cache(torch.Generator().manual_seed(6), 3, lens, Hkv, 16, "int8")
    kvq.k_tail[1] = kvq.v_tail[1] = float("nan")
    kvq.seq_lens[1] = length
    ctx = context(Hq, Hkv, batch=3, pages=kvq.block_table.shape[1])
    n = sum(new)
    q = torch.randn(n, Hq, 128, generator=torch.Generator().manual_seed(7)).to(torch.bfloat16).to(DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((n, Hq), 7.0, device=DEV)
    ctx.locks_kvq_attend(q, kvq, 3, out, lse, cu_tokens=None if n == 3 else U.cu_of(new, DEV))
    assert ctx.locks_poll_status() == 0
    check_attend(Hq, Hkv, 16, lens, new, kvq, q, out, lse)


def test_append_of_negative_lengths():
    """A new token that no length counts: reported, and nothing is written; a length of zero has no new token."""
    for length, status in ((0, 0), (-1, -6), (-2 ** 31, -6)):
        kvq = new_kvq_cache(6, 2, 2, 16, torch.arange(6, dtype=torch.int32, device=DEV).view(2, 3), torch.tensor([length, 16], dtype=torch.int32, device=DEV))
        ctx = context(4, 2, batch=2, pages=3)
        k = torch.randn(2, 2, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
        ctx.locks_kvq_append(k, k, kvq, 2)
        assert ctx.locks_poll_status() == status
        used = [int(x) for x in (kvq.k_scale.abs().sum(1) > 0).nonzero()[:, 0]]
        assert used == [3] and not bool(kvq.k_tail[0].any())


def test_append_offsets_that_go_back():
    """Offsets that give all rows to every other request: more pages than there are CTAs for, which is reported; and one request's rows out of
    range among others whose appends take place."""
    n, B, batch, heads = 160, 16, 9, 2
    k = torch.randn(n, heads, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    table = torch.arange(batch * 12, dtype=torch.int32, device=DEV).view(batch, 12)
    kvq = new_kvq_cache(batch * 12, batch, heads, B, table, torch.full((batch,), n, dtype=torch.int32, device=DEV))
    ctx = context(4, heads, batch=batch, pages=12)
    ctx.locks_kvq_append(k, k, kvq, batch, cu_tokens=torch.tensor([0 if b % 2 == 0 else n for b in range(batch + 1)], dtype=torch.int32, device=DEV))
    assert ctx.locks_poll_status() == -6
    for cu, good in (([0, 40, 90, 80, 160], [True, True, False, True]), ([0, 40, 170, 100, 160], [True, False, False, True])):
        kvq = new_kvq_cache(48, 4, heads, B, table[:4].contiguous(), torch.tensor([100, 100, 100, 100], dtype=torch.int32, device=DEV))
        ctx.locks_kvq_append(k, k, kvq, 4, cu_tokens=torch.tensor(cu, dtype=torch.int32, device=DEV))
        assert ctx.locks_poll_status() == -6
        assert [bool((kvq.k_scale.view(4, 12, heads)[b] > 0).any()) for b in range(4)] == good
    # ragged offsets that are in order: as many pages as there can be, nothing reported
    new = [17, 15, 31, 1, 33, 16, 15, 31, 1]
    kvq = new_kvq_cache(batch * 12, batch, heads, B, table, torch.tensor([m + 15 for m in new], dtype=torch.int32, device=DEV))
    ctx.locks_kvq_append(k, k, kvq, batch, cu_tokens=U.cu_of(new, DEV))
    assert ctx.locks_poll_status() == 0
    assert [int((kvq.k_scale.view(batch, 12, heads)[b, :, 0] > 0).sum()) for b in range(batch)] == [(m + 15) // 16 for m in new]
