"""CPU: what the calls around a decode step refuse before anything reaches a GPU."""
import inspect

import pytest
import torch

import paper_2607_24555_b200 as locks
from paper_2607_24555_b200 import binding


def cpu_view(**kw):
    table, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    return locks.new_kvq_cache(4, 2, 2, 16, table, lens, **kw)


@pytest.mark.parametrize("fmt,layout", [("int8", "HND"), ("e4m3", "NHD")])
def test_new_cache_has_the_layout_asked_for(fmt, layout):
    v = cpu_view(fmt=fmt, layout=layout)
    assert v.k.shape == (4, 2, 16, 128) and v.k_scale.shape == (4, 2) and v.k_tail.shape == (2, 2, 16, 128)
    assert v.k.stride() == ((4096, 2048, 128, 1) if layout == "HND" else (4096, 128, 256, 1))
    assert v.struct().fmt == (locks.KVQ_INT if fmt == "int8" else locks.KVQ_FLOAT) and v.struct().num_blocks == 4
    kv = v.kv_view()
    assert kv.num_blocks == 4 and kv.block_table is v.block_table


def test_views_refuse_what_does_not_fit():
    v = cpu_view()
    parts = dict(k=v.k, v=v.v, k_scale=v.k_scale, v_scale=v.v_scale, k_tail=v.k_tail, v_tail=v.v_tail, block_table=v.block_table, seq_lens=v.seq_lens)
    bad = dict(k=v.k.float(), v=v.v[:, :, :8], k_scale=v.k_scale.double(), v_scale=v.v_scale[:2], k_tail=v.k_tail.half(), v_tail=v.v_tail[..., :64],
               block_table=v.block_table.long(), seq_lens=v.seq_lens[None])
    locks.KVQView(**parts)
    for name, t in bad.items():
        with pytest.raises(locks.LocksError):
            locks.KVQView(**{**parts, name: t})


def test_rotary_description():
    r = locks.make_rotary([1.0, 0.5] * 16, axis=[0, 2] * 16, interleaved=True)
    assert r.rot_dim == 64 and r.num_axes == 3 and r.interleaved == 1 and list(r.axis[:4]) == [0, 2, 0, 2]
    for bad in (dict(inv_freq=[]), dict(inv_freq=[1.0] * 65), dict(inv_freq=[1.0] * 8, axis=[0] * 7), dict(inv_freq=[1.0] * 8, axis=[4] * 8), dict(inv_freq=[1.0] * 8, axis=[-1] * 8)):
        with pytest.raises(locks.LocksError):
            locks.make_rotary(**bad)


def test_native_calls_refuse_before_they_reach_the_library():
    """A context without a library handle behind it: every refusal has to come before the handle is used."""
    m = binding.calls()
    ctx = m.context(1, 4, 2, 2, 4, 16, 2, 0, False, 832, True)
    q, k = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 2, 128, dtype=torch.bfloat16)
    rot = locks.make_rotary([1.0] * 64)
    pos = torch.zeros(1, 2, dtype=torch.int32)
    v = cpu_view()
    calls = [
        (m.rope, (ctx, rot, pos, q, q, None, None, None), "cuda:0"),
        (m.rope, (ctx, rot, None, q, q, None, None, None), "needed"),
        (m.rope, (ctx, rot, pos, q, None, None, None, None), "q_out"),
        (m.rope, (ctx, rot, pos, None, None, None, None, None), "q_out"),
        (m.rope, (ctx, rot, pos, "q", q, None, None, None), "no tensor"),
        (m.rope, (ctx, b"short", pos, q, q, None, None, None), "make_rotary"),
        (m.append_rows, (ctx, k, k, v.kv_view(), 3, None, None, None, None, None, None), "batch"),
        (m.append_rows, (ctx, k, k, v.kv_view(), 2, None, None, q, q, None, None), "rotary"),
        (m.kvq_append, (ctx, k, k, v, 2, rot, pos, q, None, None, None), "q_out"),
        (m.kvq_append, (ctx, k, k, v, 2, None, None, None, None, None, None), "cuda:0"),
        (m.kvq_attend, (ctx, q, v, 0, q, None, None, None, None, None), "batch"),
        (m.kvq_attend, (ctx, q, v, 2, q, None, None, None, None, None), "cuda:0"),
        (m.kvq_build_summaries, (ctx, v, 2, torch.zeros(1, dtype=torch.uint8), None, None, None), "cuda:0"),
    ]
    for f, args, word in calls:
        with pytest.raises(locks.LocksError, match=word):
            f(*args)
    with pytest.raises(TypeError):
        m.rope(ctx)
    m.close(ctx)
    with pytest.raises(locks.LocksError, match="closed"):
        m.rope(ctx, rot, pos, q, q, None, None, None)


def test_library_refuses_bad_arguments_without_a_context():
    """The C entry points themselves, by ctypes: no context, nothing launched."""
    import ctypes as C
    L = binding.lib()
    r, rows = locks.make_rotary([1.0] * 64), binding.Rows(256, 128, 128)
    assert L.locks_rope(None, C.byref(r), 256, 1, C.byref(rows), C.byref(rows), None, None, None) == -1
    assert L.locks_append_rows(None, None, None, None, 1, None, None, C.byref(rows), C.byref(rows), None, 1, None) == -1
    assert L.locks_kvq_append(None, None, None, None, 1, None, None, C.byref(rows), C.byref(rows), None, 1, None) == -1
    assert L.locks_kvq_attend(None, None, None, 1, None, 1, None, None, None, None, None) == -1
    assert L.locks_kvq_build_summaries(None, None, 1, None, None, None, None) == -1


def test_the_view_for_the_selector_is_no_cache():
    """Codes are one byte each: a call that took the view for rows of the configuration's type would read beyond them."""
    view = cpu_view().kv_view()
    assert view.tables().seq_lens == view.seq_lens.data_ptr() and view.tables().num_blocks == 4
    with pytest.raises(locks.LocksError, match="reads keys"):
        view.struct()
    reads = ["locks_build_summaries", "locks_sparse_attend", "locks_decode_step", "locks_decode_step_host", "locks_select_exact", "locks_select_rival",
             "locks_fake_quantize_pages", "locks_build_summaries_layers"]
    ctx = object.__new__(locks.Context)
    ctx.handle = None
    for name in reads:
        call = getattr(ctx, name)
        args = {p: view if p == "kv" else ([torch.zeros(1)] if p.endswith("_layers") else None) for p in inspect.signature(call).parameters}
        if "scorer" in args:
            args["scorer"] = 1
        with pytest.raises(locks.LocksError, match="reads keys"):
            call(**args)
    with pytest.raises(locks.LocksError, match="reads keys"):
        locks.locks_sparse_attend_noalloc(binding.make_config(4, 2, 8, "i4", "bf16", 2, 4, 32), None, view, 2, None, None, None)


def test_tails_of_one_or_two_pages():
    for pages in (1, 2):
        v = cpu_view(tail_pages=pages)
        assert v.k_tail.shape == (2, 2, 16 * pages, 128) and v.tail_pages == pages and v.struct().tail_pages == pages
    two, one = cpu_view(tail_pages=2), cpu_view()
    parts = dict(k=two.k, v=two.v, k_scale=two.k_scale, v_scale=two.v_scale, block_table=two.block_table, seq_lens=two.seq_lens)
    with pytest.raises(locks.LocksError, match="one size"):
        locks.KVQView(k_tail=two.k_tail, v_tail=one.v_tail, **parts)
    three = torch.zeros(2, 2, 48, 128)
    with pytest.raises(locks.LocksError, match="twice"):
        locks.KVQView(k_tail=three, v_tail=three, **parts)
