"""GPU: rotations and appends followed, on one stream and without a pause, by the calls that read what they wrote."""
import pytest
import torch

import kvq_util as U
import paper_2607_24555_b200 as locks
from paper_2607_24555_b200.binding import KVView, make_config, make_rotary
from test_gpu_kvq import DEV, freqs, rows

pytestmark = pytest.mark.gpu


class Layer:
    """A layer with a bf16 cache of random rows; q is rotated into qo, which starts as anything."""

    def __init__(self, Hq, Hkv, B, batch, T, budget, seed=0, fill_summaries=False):
        gen = torch.Generator().manual_seed(seed)
        self.Hq, self.Hkv, self.batch = Hq, Hkv, batch
        pages = T // B + 8
        nb = batch * pages
        self.cache = [torch.randn(nb, Hkv, B, 128, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2)]
        table = torch.randperm(nb, generator=gen).to(torch.int32).view(batch, pages).to(DEV)
        self.seq = torch.full((batch,), T, dtype=torch.int32, device=DEV)
        self.kv = KVView(*self.cache, self.cache[0].stride()[:3], nb, table, self.seq)
        self.ctx = locks.Context(make_config(Hq, Hkv, 8, "i4", "bf16", batch, pages, budget, B=B), device=DEV)
        self.q, self.k, self.v = rows(gen, batch, Hq, "bf16"), rows(gen, batch, Hkv, "bf16"), rows(gen, batch, Hkv, "bf16")
        self.qo, self.out = torch.zeros_like(self.q), torch.zeros_like(self.q)
        self.rot, self.gen = make_rotary(freqs(128)), gen
        self.pos = self.seq - 1
        self.ids = torch.zeros(batch, Hkv, self.ctx.k, dtype=torch.int32, device=DEV)
        self.cnt = torch.zeros(batch, Hkv, dtype=torch.int32, device=DEV)
        self.summ = self.ctx.new_summaries(nb)
        if fill_summaries:
            self.ctx.locks_build_summaries(self.kv, batch, self.summ)

    def append(self):
        self.ctx.locks_append_rows(self.k, self.v, self.kv, self.batch, rotary=self.rot, q=self.q, q_out=self.qo)

    def rope(self):
        self.ctx.locks_rope(self.rot, self.pos, self.q, self.qo)

    def dense(self):
        self.ctx.locks_sparse_attend(self.qo, self.kv, self.batch, None, None, self.out)

    def listed(self):
        self.ctx.locks_sparse_attend(self.qo, self.kv, self.batch, self.ids, self.cnt, self.out)

    def exact(self):
        self.ctx.locks_select_exact(self.qo, self.kv, self.batch, self.ids, self.cnt)

    def select(self):
        self.ctx.locks_select(self.qo, self.summ, self.kv, self.batch, self.ids, self.cnt)

    def step(self):
        self.ctx.locks_decode_step(self.qo, None, None, self.kv, self.summ, self.batch, self.out, self.ids, self.cnt)


def check_in_turn(layer, calls, turns=12):
    """Captured and replayed with new queries each time: bit for bit what the calls give with a pause after each."""
    def run(pause):
        for c in calls:
            getattr(layer, c)()
            if pause:
                torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(True)
        with torch.cuda.graph(graph, stream=side):
            run(False)
        for turn in range(turns):
            for t, heads in ((layer.q, layer.Hq), (layer.k, layer.Hkv), (layer.v, layer.Hkv)):
                t.copy_(rows(layer.gen, layer.batch, heads, "bf16"))
            got = []
            for paused in (False, True):
                for t in (layer.out, layer.ids, layer.cnt):
                    t.zero_()
                layer.qo.fill_(3.0)   # an old query
                side.synchronize()
                if paused:
                    run(True)
                else:
                    graph.replay()
                side.synchronize()
                got.append([t.clone() for t in (layer.out, layer.ids, layer.cnt, layer.qo)])
            for a, b in zip(*got):
                assert torch.equal(a, b), (calls, turn)
    torch.cuda.current_stream().wait_stream(side)
    assert layer.ctx.locks_poll_status() == 0


@pytest.mark.parametrize("Hq,Hkv,B,batch,T", [(32, 8, 16, 8, 800), (32, 2, 16, 1, 200), (8, 2, 32, 5, 333), (28, 4, 64, 33, 130)])
@pytest.mark.parametrize("write", ["append", "rope"])
def test_rotated_queries_are_there_for_dense_attention(Hq, Hkv, B, batch, T, write):
    check_in_turn(Layer(Hq, Hkv, B, batch, T, 4 * B), [write, "dense"])


@pytest.mark.parametrize("Hq,Hkv,batch,T", [(32, 8, 8, 1500), (32, 2, 3, 3000)])
@pytest.mark.parametrize("write", ["append", "rope"])
def test_rotated_queries_are_there_for_the_exact_selector(Hq, Hkv, batch, T, write):
    layer = Layer(Hq, Hkv, 16, batch, T, 256)
    check_in_turn(layer, [write, "exact"])
    check_in_turn(layer, [write, "exact", "listed"])
    check_in_turn(layer, [write, "listed"])   # a page table that is there already


@pytest.mark.parametrize("Hq,Hkv,B,batch,T,budget", [(32, 8, 16, 1, 2000, 256), (32, 8, 16, 8, 2000, 512), (32, 8, 16, 16, 1000, 256), (32, 2, 16, 8, 2000, 512),
                                                     (32, 8, 32, 4, 2000, 512), (32, 8, 16, 32, 700, 256), (32, 8, 16, 64, 700, 256)])
def test_rotated_queries_are_there_for_a_decode_step(Hq, Hkv, B, batch, T, budget):
    """Batches on both sides of the rule that lets a step's attention start beside its selector."""
    layer = Layer(Hq, Hkv, B, batch, T, budget, fill_summaries=True)
    check_in_turn(layer, ["append", "step"])
    check_in_turn(layer, ["rope", "step"])
    check_in_turn(layer, ["append", "select", "listed"])


def test_many_layers_in_one_graph():
    """Eight layers, each append, attention and the next layer's rotation: no pause anywhere."""
    layers = [Layer(32, 8, 16, 8, 500 + 100 * i, 256, seed=i) for i in range(8)]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())

    def run(pause):
        for l in layers:
            l.append()
            if pause:
                torch.cuda.synchronize()
            l.dense()
            if pause:
                torch.cuda.synchronize()
    with torch.cuda.stream(side):
        run(True)
        with torch.cuda.graph(graph, stream=side):
            run(False)
        for turn in range(10):
            for l in layers:
                l.q.copy_(rows(l.gen, l.batch, l.Hq, "bf16"))
            graph.replay()
            side.synchronize()
            got = [l.out.clone() for l in layers]
            run(True)
            for l, o in zip(layers, got):
                assert torch.equal(l.out, o), turn
    torch.cuda.current_stream().wait_stream(side)


def test_contexts_do_without_the_native_call_layer(monkeypatch, tmp_path):
    from paper_2607_24555_b200 import binding
    monkeypatch.setattr(binding, "_CALLS_PATH", str(tmp_path / "_calls.so"))
    monkeypatch.setattr(binding, "_calls_module", None)
    layer = Layer(8, 2, 16, 2, 100, 64, fill_summaries=True)
    layer.qo.copy_(layer.q)
    layer.step()
    torch.cuda.synchronize()
    assert layer.ctx.locks_poll_status() == 0 and bool(torch.isfinite(layer.out.float()).all())
    with pytest.raises(locks.LocksError, match="missing"):
        layer.rope()
    layer.ctx.close()
    with pytest.raises(locks.LocksError, match="closed"):
        layer.rope()
