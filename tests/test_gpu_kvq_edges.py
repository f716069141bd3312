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
    ctx = context(Hq, Hkv, batch=3, pages=kvq.block_table.shape[1])
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
    ctx = context(Hq, Hkv, B=B, batch=1, pages=kvq.block_table.shape[1])
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
    ctx = context(Hq, Hkv, batch=len(lens), pages=kvq.block_table.shape[1])
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
