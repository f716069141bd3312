"""GPU: drafted tokens in the 8-bit cache that are refused: a sequence is shortened, attended and appended to again, and is then what a
cache holds that never saw them, bit for bit."""
import ctypes as C

import pytest
import torch

import kvq_util as U
from paper_2607_24555_b200 import binding
from paper_2607_24555_b200.binding import make_rotary, new_kvq_cache
from test_gpu_kvq import DEV, context, freqs, rows

pytestmark = pytest.mark.gpu
Hq, Hkv = 8, 2


class Cache:
    def __init__(self, B, batch, pages, fmt, layout="HND", tail_pages=1):
        table = torch.arange(batch * pages, dtype=torch.int32, device=DEV).view(batch, pages)
        self.kvq = new_kvq_cache(batch * pages, batch, Hkv, B, table, torch.zeros(batch, dtype=torch.int32, device=DEV), fmt=fmt, layout=layout, tail_pages=tail_pages)
        self.kvq.k_tail.fill_(float("nan"))   # (nothing that was not appended may be used)
        self.kvq.v_tail.fill_(float("nan"))
        self.ctx = context(Hq, Hkv, B=B, batch=batch, pages=pages, budget=2 * B)
        self.B, self.batch, self.rot = B, batch, make_rotary(freqs(128))

    def set(self, lens):
        self.kvq.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))

    def append(self, k, v, lens, new):
        """The sequences' rows lens[b] - new[b] .. of k[b], v[b]."""
        self.set(lens)
        part = [torch.cat([x[b][t - m:t] for b, (t, m) in enumerate(zip(lens, new))]) for x in (k, v)]
        if part[0].shape[0]:
            self.ctx.locks_kvq_append(*part, self.kvq, self.batch, rotary=self.rot, cu_tokens=U.cu_of(new, DEV))

    def attend(self, q, lens, new):
        self.set(lens)
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
        self.ctx.locks_kvq_attend(q, self.kvq, self.batch, out, lse, cu_tokens=U.cu_of(new, DEV))
        return out, lse


def check_alike(a, c, lens, gen, what):
    """Codes, scales and rows of the unfinished pages, and attention of one and of several tokens, bit for bit."""
    B = a.B
    for b, t in enumerate(lens):
        blocks = a.kvq.block_table[b, :t // B].long()
        for n in ("k", "v"):
            assert torch.equal(getattr(a.kvq, n)[blocks].view(torch.uint8), getattr(c.kvq, n)[blocks].view(torch.uint8)), (what, b, n)
            assert torch.equal(getattr(a.kvq, n + "_scale")[blocks], getattr(c.kvq, n + "_scale")[blocks]), (what, b, n)
            x, y = [getattr(o.kvq, n + "_tail")[b, :, t // B % o.kvq.tail_pages * B:][:, :t % B] for o in (a, c)]
            assert torch.equal(x, y), (what, b, n)
    for new in ([1] * a.batch, [min(3, t) for t in lens]):
        if not any(new):
            continue
        q = rows(gen, sum(new), Hq, "bf16")
        for x, y in zip(a.attend(q, lens, new), c.attend(q, lens, new)):
            assert torch.equal(x, y) and not bool(torch.isnan(x.float()).any()), what


@pytest.mark.parametrize("fmt,layout", [("int8", "HND"), ("e4m3", "NHD")])
@pytest.mark.parametrize("B", [16, 32, 64])
def test_refused_drafts_leave_nothing(B, fmt, layout):
    """Rounds of up to eight drafts of three requests, of which some, none or all stay; pages end at every place of them."""
    gen = torch.Generator().manual_seed(B)
    batch, longest = 3, 5 * B + 11
    k, v = [[rows(gen, longest + 8, Hkv, "bf16") for _ in range(batch)] for _ in range(2)]
    pages = (longest + 8) // B + 2
    a, c = Cache(B, batch, pages, fmt, layout, tail_pages=2), Cache(B, batch, pages, fmt, layout)
    lens = [2 * B - 3, B + 1, 5]
    for o in (a, c):
        o.append(k, v, lens, lens)
    while min(lens) < longest:
        drafts = [min(int(torch.randint(1, 9, (1,), generator=gen)), longest + 8 - t) if t < longest else 0 for t in lens]
        stay = [int(torch.randint(0, d + 1, (1,), generator=gen)) for d in drafts]
        # drafts: other rows than those that will be the sequence's, but for the ones that stay
        wrong = [[torch.cat([x[b][:t + s], rows(gen, d - s, Hkv, "bf16"), x[b][t + d:]]) if d else x[b] for b, (t, d, s) in enumerate(zip(lens, drafts, stay))] for x in (k, v)]
        a.append(*wrong, [t + d for t, d in zip(lens, drafts)], drafts)
        lens = [t + s for t, s in zip(lens, stay)]
        c.append(k, v, lens, stay)
        check_alike(a, c, lens, gen, (lens, drafts, stay))
    assert a.ctx.locks_poll_status() == 0 and c.ctx.locks_poll_status() == 0


@pytest.mark.parametrize("B", [16, 32, 64])
@pytest.mark.parametrize("before,upto", [(0, 150), (5, 150), (37, 167), (37, 128), (16, 256), (90, 100), (1, 65), (33, 34), (7, 135)])
def test_a_prompt_is_shortened_by_up_to_a_page(B, before, upto):
    """Appends over many pages (the tail's page of the first of them is that of a later one, too), then any length that is allowed."""
    gen = torch.Generator().manual_seed(upto)
    k, v = [[rows(gen, upto + B, Hkv, "bf16")] for _ in range(2)]
    pages = (upto + B) // B + 2
    low = max((upto // B - 1) * B, 0)
    for back in sorted({low, low + 1, low + B // 2, low + B - 1, upto // B * B, upto - 1, upto}):
        if not low <= back <= upto:
            continue
        a, c = Cache(B, 1, pages, "int8", tail_pages=2), Cache(B, 1, pages, "int8")
        for o in (a, c):
            o.append(k, v, [before], [before])
        a.append(k, v, [upto], [upto - before])
        c.append(k, v, [min(before, back)], [0])
        if back >= before:
            c.append(k, v, [back], [back - before])
        else:   # (into the rows before)
            c = Cache(B, 1, pages, "int8")
            c.append(k, v, [back], [back])
        check_alike(a, c, [back], gen, (before, upto, back))
        # and on from there with other rows
        on = [[torch.cat([x[0][:back], rows(gen, upto + B - back, Hkv, "bf16")])] for x in (k, v)]
        for o in (a, c):
            o.append(*on, [back + B - 2], [B - 2])
        check_alike(a, c, [back + B - 2], gen, (before, upto, back, "on"))


def test_one_tail_page_and_a_copy_of_it():
    """The way that include/locks.h gives for caches with one tail page: the tail from before the drafts, and the tokens that stay again."""
    B, gen = 16, torch.Generator().manual_seed(4)
    k, v = [[rows(gen, 80, Hkv, "bf16") for _ in range(2)] for _ in range(2)]
    a, c = Cache(B, 2, 6, "int8"), Cache(B, 2, 6, "int8")
    lens, drafts, stay = [30, 45], [6, 7], [1, 2]   # both complete a page; what stays does so for the second only by one
    for o in (a, c):
        o.append(k, v, lens, lens)
    copy = [getattr(a.kvq, n).clone() for n in ("k_tail", "v_tail")]
    a.append(k, v, [36, 52], drafts)
    for n, t in zip(("k_tail", "v_tail"), copy):
        getattr(a.kvq, n).copy_(t)
    lens = [31, 47]
    for o in (a, c):
        o.append(k, v, lens, stay)
    check_alike(a, c, lens, gen, "copy")


@pytest.mark.parametrize("m", [1, 40])
def test_captured_drafts(m):
    """Append and attention captured once; lengths set back between the replays."""
    B, gen, batch = 16, torch.Generator().manual_seed(m), 2
    k, v = [[rows(gen, 700, Hkv, "bf16") for _ in range(batch)] for _ in range(2)]
    a, c = Cache(B, batch, 50, "e4m3", tail_pages=2), Cache(B, batch, 50, "e4m3")
    lens = [41, 90]
    for o in (a, c):
        o.append(k, v, lens, lens)
    kk, vv, cu = rows(gen, m * batch, Hkv, "bf16"), rows(gen, m * batch, Hkv, "bf16"), U.cu_of([m] * batch, DEV)
    q = rows(gen, m * batch, Hq, "bf16")
    out = torch.empty_like(q)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            a.kvq.seq_lens += m
            a.ctx.locks_kvq_append(kk, vv, a.kvq, batch, rotary=a.rot, cu_tokens=cu)
            a.ctx.locks_kvq_attend(q, a.kvq, batch, out, cu_tokens=cu)
        for turn in range(8):
            a.set(lens)
            for t, x in ((kk, k), (vv, v)):
                t.copy_(torch.cat([x[b][n:n + m] for b, n in enumerate(lens)]))
            graph.replay()
            stay = [max(m - turn % 17, 0), m]
            lens = [n + s for n, s in zip(lens, stay)]
            c.append(k, v, lens, stay)
            check_alike(a, c, lens, gen, (m, turn))
    torch.cuda.current_stream().wait_stream(side)


@pytest.mark.parametrize("B", [16, 32, 64])
@pytest.mark.parametrize("lens", [[150, 203], [128 + 31, 64 + 17], [192, 255]])
def test_chunks_find_the_tail(lens, B):
    """The many-row form, unfinished pages in either page of the tail; an infinite value in one of them."""
    gen = torch.Generator().manual_seed(B)
    k, v = [[rows(gen, t, Hkv, "bf16") for t in lens] for _ in range(2)]
    a, c = Cache(B, 2, 20, "int8", tail_pages=2), Cache(B, 2, 20, "int8")
    before, new = [t // 3 for t in lens], [min(t, 100) for t in lens]
    for o in (a, c):
        o.append(k, v, before, before)
        o.append(k, v, lens, [t - n for t, n in zip(lens, before)])
    q = rows(gen, sum(new), Hq, "bf16")
    assert sum(new) * 4 >= 96 * 2 and sum(new) * Hq >= 768
    for turn in range(2):
        got = [o.attend(q, lens, new) for o in (a, c)]
        for x, y in zip(*got):
            assert torch.equal(x, y) and not bool(torch.isnan(x.float()).any())
        assert bool(torch.isfinite(got[0][0].float()).all()) == (turn == 0 or lens[0] % B == 0)
        for o in (a, c):
            o.kvq.v_tail[0, 1, lens[0] // B % o.kvq.tail_pages * B, 5] = float("inf")


def test_tails_of_other_sizes_are_refused():
    a = Cache(16, 1, 4, "int8")
    s = a.kvq.struct()
    assert s.tail_pages == 1
    k = rows(torch.Generator().manual_seed(0), 1, Hkv, "bf16")
    r = binding.Rows(k.data_ptr(), k.stride(0), k.stride(1))
    for pages, rc in ((3, -1), (-1, -1), (0, 0), (1, 0)):   # (0: as 1)
        s.tail_pages = pages
        assert binding.lib().locks_kvq_append(a.ctx.handle, None, None, None, 1, None, None, C.byref(r), C.byref(r), C.byref(s), 1, None) == rc
    torch.cuda.synchronize()
