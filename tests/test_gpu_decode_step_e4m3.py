"""SparseDecodeStep over an e4m3 cache: a few decode steps equal the separate calls bit for bit, in a
graph too, and stay near the bf16 step on the values that the cache holds."""
import numpy as np
import pytest
import torch

import e4m3
from paper_2606_08446_amd import sparrow as S
from paper_2606_08446_amd import workloads as W

from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
D = 128


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


class Layer:
    """A layer with prompts in its e4m3 cache, room for a few tokens, and its step."""

    def __init__(self, seed, G, landmark, prompts=(300, 1000, 17), steps=4, **kw):
        g = torch.Generator().manual_seed(seed)
        hkv, ps, B = 2, 16, len(prompts)
        pages = [(n + steps) // ps + 1 for n in prompts]
        perm, at = torch.randperm(sum(pages), generator=g).to(torch.int32), 0
        bt = torch.zeros((B, max(pages)), dtype=torch.int32)
        for b, n in enumerate(pages):
            bt[b, :n] = perm[at:at + n]
            at += n
        self.bt = bt.to(DEV)
        self.k8, self.v8, self.exps = S.new_cache_e4m3(sum(pages), hkv, ps, DEV)
        self.meta = S.new_meta(sum(pages), hkv, DEV, landmark)
        T = sum(prompts)
        cu = torch.tensor(np.concatenate([[0], np.cumsum(prompts)]), dtype=torch.int32, device=DEV)
        rows = [torch.randn((T, hkv, D), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2)]
        self.lens = torch.tensor(prompts, dtype=torch.int32, device=DEV)
        S.append_kv_e4m3(rows[0], rows[1], self.k8, self.v8, self.exps, self.bt, self.lens,
                         self.meta, cu_tokens=cu, landmark=landmark)
        # new rows inside a fused projection's output
        qkv = torch.randn((steps, B, 2 * hkv * D), generator=g).to(torch.bfloat16).to(DEV)
        self.k_new = qkv[..., :hkv * D].unflatten(2, (hkv, D))
        self.v_new = qkv[..., hkv * D:].unflatten(2, (hkv, D))
        self.q = torch.randn((B, G * hkv, D), generator=g).to(torch.bfloat16).to(DEV)
        table = torch.tensor([2], dtype=torch.int32, device=DEV)
        frac = torch.tensor([200], dtype=torch.int32, device=DEV)
        self.landmark, self.tables = landmark, (table, frac, 1000, 2048, 16)
        self.kw = kw
        self.step = S.SparseDecodeStep(self.q, self.k8, self.v8, self.bt, self.lens, self.meta,
                                       *self.tables, landmark=landmark, exps=self.exps, **kw)

    def state(self):
        return [t.view(torch.uint8).clone() for t in (self.k8, self.v8, self.exps, self.meta)]

    def restore(self, state):
        for t, s in zip((self.k8, self.v8, self.exps, self.meta), state):
            t.view(torch.uint8).copy_(s)


CASES = [(4, 0, {}), (10, 0, {}), (4, S.SPARROW_LANDMARK_MEAN, dict(sink_pages=1, local_pages=2))]


@pytest.mark.parametrize("G,landmark,kw", CASES)
def test_steps_equal_the_separate_calls(G, landmark, kw):
    log(f"case e4m3 step G={G} landmark={landmark}")
    a, b = Layer(5, G, landmark, **kw), Layer(5, G, landmark, **kw)
    stream = torch.cuda.current_stream().cuda_stream
    for i in range(4):
        lens = a.lens + 1 + i
        if i % 2:
            a.step.decode_step(a.k_new[i], a.v_new[i], stream, seq_lens=lens)
        else:
            a.step.append_score_topk(a.k_new[i], a.v_new[i], stream, seq_lens=lens)
            a.step.attend(stream, seq_lens=lens)
        S.append_kv_e4m3(b.k_new[i], b.v_new[i], b.k8, b.v8, b.exps, b.bt, lens, b.meta,
                         landmark=landmark)
        k, idx = S.page_score_topk(b.q, b.meta, b.bt, lens, b.k8.shape, *b.tables,
                                   landmark=landmark, **kw)
        out = S.sparse_decode_attn_e4m3(b.q, b.k8, b.v8, b.exps, b.bt, lens, k, idx)
        assert torch.equal(a.step.k, k) and torch.equal(a.step.idx, idx) and \
            torch.equal(a.step.out, out), i
        assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state())), i
    # without an append: the same step again
    again = a.step.out.clone()
    assert torch.equal(a.step.decode_step(None, None, stream, seq_lens=lens), again)
    # the bf16 step on the same values: its numerators have 8 bits (2^-8 of sum w |v| <= max |v|)
    kv, vv = e4m3.both_values(a.k8, a.v8, a.exps)
    kb, vb = (torch.from_numpy(x).to(torch.bfloat16).to(DEV) for x in (kv, vv))
    ref = S.sparse_decode_attn(a.q, kb, vb, a.bt, lens, a.step.k, a.step.idx)
    assert float((ref - a.step.out).abs().max()) <= 2.0 ** -7 * float(np.abs(vv).max())


def test_layers_in_a_graph():
    layers = [Layer(20 + i, 4 if i % 2 else 10, 0) for i in range(3)]
    lens = [x.lens + 1 for x in layers]
    before = [x.state() for x in layers]
    stream = torch.cuda.current_stream().cuda_stream
    for x, n in zip(layers, lens):
        x.step.decode_step(x.k_new[0], x.v_new[0], stream, seq_lens=n)
    want = [(x.step.out.clone(), x.step.idx.clone(), x.state()) for x in layers]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        for x, n in zip(layers, lens):
            x.step.decode_step(x.k_new[0], x.v_new[0], side.cuda_stream, seq_lens=n)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(3):
        for x, s in zip(layers, before):
            x.restore(s)
            x.step.out.fill_(7)
            x.step.idx.fill_(-5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, (out, idx, state) in zip(layers, want):
            assert torch.equal(x.step.out, out) and torch.equal(x.step.idx, idx), rep
            assert all(torch.equal(p, r) for p, r in zip(x.state(), state)), rep


def test_refusals():
    x = Layer(9, 4, 0)
    stream = torch.cuda.current_stream().cuda_stream
    args = (x.q, x.k8, x.v8, x.bt, x.lens, x.meta) + x.tables
    with pytest.raises(ValueError):
        S.SparseDecodeStep(*args)                                   # e4m3 caches without exps
    with pytest.raises(ValueError):
        S.SparseDecodeStep(*args, exps=x.exps[:1])
    with pytest.raises(ValueError):
        S.SparseDecodeStep(x.q.float(), *args[1:], exps=x.exps)
    with pytest.raises(ValueError):
        x.step.meta_update(None, stream)
    with pytest.raises(ValueError):
        x.step.run(first_pos=x.lens - 1)
    with pytest.raises(ValueError):
        x.step.append(x.k_new[0].float(), x.v_new[0], stream)
    with pytest.raises(ValueError):
        x.step.decode_step(x.k_new[0], None, stream)
    w = W.small()
    inp = W.generate(w, DEV, lengths=[40, 70])
    with pytest.raises(ValueError):                                 # bf16 caches with exps
        S.SparseDecodeStep(inp.q, inp.k_cache, inp.v_cache, inp.block_table, inp.seq_lens,
                           S.new_meta(inp.num_phys_pages, 2, DEV), *x.tables, exps=x.exps)
