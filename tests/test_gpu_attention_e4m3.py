"""Decode attention over an e4m3 cache against the formula in 64 bits.

Tolerance of an output, in units of sum_t w_t |v_t|: a logit is a sum of 128 exact products in fp32,
off by at most 2^-17 of scale sum |q k| (128 steps of 2^-24), and so is a weight's logarithm, once in
the numerator and once in the sum: 2 * 2^-17 * max_t scale sum |q k_t|.  The numerators have 17 bits
(2^-17), exp2 and the running maximum's corrections a few steps of 2^-24 each tile; the sums run over at
most a few hundred tiles per wave and as many partials: 2^-14 covers them.  Then one rounding to the
output's type: 2^-8 of the value for bf16."""
import math

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
SCALE = 1 / math.sqrt(D)


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


class Case:
    def __init__(self, seed, lens, hq, hkv, ps, spread=0, absent=()):
        g = np.random.default_rng(seed)
        self.hq, self.hkv, self.ps, self.lens = hq, hkv, ps, np.array(lens, np.int64)
        pages = np.maximum(0, -(-self.lens // ps)) + 1
        P = int(pages.sum())
        perm = g.permutation(P)
        bt = np.full((len(lens), int(pages.max())), -1, np.int32)
        at = 0
        for b, n in enumerate(pages):
            bt[b, :n] = perm[at:at + n]
            at += n
        for b, p, phys in absent:
            bt[b, p] = phys
        self.bt_host = bt
        self.k8, self.v8, self.exps = S.new_cache_e4m3(P, hkv, ps, DEV)
        for j, c in enumerate((self.k8, self.v8)):
            x = g.standard_normal((P, hkv, ps, D))
            if spread:        # rows of different sizes
                x = np.ldexp(x, g.integers(-spread, spread + 1, (P, hkv, ps, 1)))
            y, e = e4m3.quantise(x)
            c.copy_(torch.from_numpy(y).float().to(DEV))
            self.exps[:, :, :, j] = torch.from_numpy(e + 127).to(torch.uint8).view(
                P, hkv, ps // 4, 4).to(DEV)
        self.kv, self.vv = e4m3.both_values(self.k8, self.v8, self.exps)
        self.q = torch.from_numpy(g.standard_normal((len(lens), hq, D))).to(torch.bfloat16).to(DEV)
        self.bt = torch.from_numpy(bt).to(DEV)
        self.seq_lens = torch.from_numpy(self.lens.astype(np.int32)).to(DEV)
        self.g = g

    def poison(self):
        """NaN codes and the largest exponent in every slot past the lengths and in spare pages."""
        live = np.zeros(self.kv.shape[:3], bool)
        for b, L in enumerate(self.lens):
            for p in range(min(max(0, -(-int(L) // self.ps)), self.bt_host.shape[1])):
                if 0 <= self.bt_host[b, p] < live.shape[0]:
                    live[self.bt_host[b, p], :, :min(self.ps, int(L) - p * self.ps)] = True
        dead = torch.from_numpy(~live).to(DEV)
        for j, c in enumerate((self.k8, self.v8)):
            c.view(torch.uint8)[dead] = 0x7f
            e = self.exps[:, :, :, j].reshape(dead.shape)
            e[dead] = 255
            self.exps[:, :, :, j] = e.view(dead.shape[0], self.hkv, -1, 4)

    def lists(self, counts, k_max, sort=True):
        idx = np.full((len(self.lens), self.hkv, k_max), -1, np.int32)
        for b, L in enumerate(self.lens):
            n = max(0, -(-int(L) // self.ps))
            for h in range(self.hkv):
                pick = self.g.permutation(n)[:counts[b]]
                idx[b, h, :len(pick)] = np.sort(pick) if sort else pick
        return idx

    def formula(self, idx=None, k=None, scale=SCALE):
        """(output, sum w |v|, largest scale sum |q k|) in 64 bits, [B][Hq][128] and [B][Hq]."""
        B, G, P = len(self.lens), self.hq // self.hkv, self.kv.shape[0]
        q = self.q.float().cpu().numpy().astype(np.float64)
        out, size, far = np.zeros((B, self.hq, D)), np.zeros((B, self.hq, D)), np.zeros((B, self.hq))
        M = self.bt_host.shape[1]
        for b in range(B):
            L = min(max(0, int(self.lens[b])), M * self.ps)
            n = -(-L // self.ps)
            for h in range(self.hkv):
                pages = range(n) if idx is None else \
                    [int(p) for p in idx[b, h, :max(0, min(int(k[b]), idx.shape[2]))]]
                at = [(int(self.bt_host[b, p]), t) for p in pages if 0 <= p < n
                      and 0 <= self.bt_host[b, p] < P
                      for t in range(min(self.ps, L - p * self.ps))]
                if not at:
                    continue
                ph, sl = np.array(at).T
                K, V = self.kv[ph, h, sl], self.vv[ph, h, sl]
                for j in range(h * G, (h + 1) * G):
                    z = scale * (K @ q[b, j])
                    w = np.exp(z - z.max())
                    w /= w.sum()
                    out[b, j], size[b, j] = w @ V, w @ np.abs(V)
                    far[b, j] = abs(scale) * (np.abs(K) @ np.abs(q[b, j])).max()
        return out, size, far

    def check(self, got, want, what):
        out, size, far = want
        g = got.float().cpu().numpy().astype(np.float64)
        tol = (2.0 ** -16 * far[..., None] + 2.0 ** -14) * size
        tol += np.abs(out) * (2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24)
        over = np.abs(g - out) - tol
        assert (over <= 0).all(), (what, float(over.max()), float(np.abs(g - out).max()))
        assert (g[size.sum(-1) == 0] == 0).all()


def dense(c, **kw):
    return S.dense_decode_attn_e4m3(c.q, c.k8, c.v8, c.exps, c.bt, c.seq_lens, **kw)


def sparse(c, k, idx, **kw):
    return S.sparse_decode_attn_e4m3(c.q, c.k8, c.v8, c.exps, c.bt, c.seq_lens,
                                     torch.tensor(k, dtype=torch.int32, device=DEV),
                                     torch.from_numpy(idx).to(DEV), **kw)


LENS = [1, 0, 15, 16, 17, 31, 33, 64, 100, 129, 700, -3]


@pytest.mark.parametrize("ps", [16, 32, 64, 128])
@pytest.mark.parametrize("hq,hkv", [(8, 8), (6, 3), (16, 4), (10, 2), (16, 1)])
@pytest.mark.parametrize("dt", [S.SPARROW_OUT_F32, S.SPARROW_OUT_BF16])
def test_dense(ps, hq, hkv, dt):
    log(f"case e4m3 dense ps={ps} heads={hq},{hkv} dt={dt}")
    c = Case(ps + hq, LENS, hq, hkv, ps)
    c.poison()
    c.check(dense(c, out_dtype=dt), c.formula(), "dense")


@pytest.mark.parametrize("lens", [[1], [5000], [4097, 3], [1000] * 40, [0, 0], [16]])
def test_dense_lengths(lens):
    log(f"case e4m3 dense lengths {lens[:4]} x {len(lens)}")
    c = Case(len(lens), lens, 16, 2, 16)
    c.poison()
    c.check(dense(c), c.formula(), lens[:4])


def test_dense_longer_than_the_table_and_absent_pages():
    c = Case(3, [300, 90, 64, 33], 4, 2, 16,
             absent=[(0, 0, -1), (0, 7, 1 << 30), (1, 5, -5), (2, 0, 1 << 29), (2, 1, -1),
                     (2, 2, -1), (2, 3, -1)])
    c.lens[3] = c.bt_host.shape[1] * 16 + 99     # its further pages are absent
    c.seq_lens[3] = int(c.lens[3])
    c.poison()
    got = dense(c)
    c.check(got, c.formula(), "absent")
    assert bool((got[2] == 0).all())


@pytest.mark.parametrize("ps", [16, 32, 64, 128])
@pytest.mark.parametrize("hq,hkv", [(8, 4), (32, 2)])
def test_sparse(ps, hq, hkv):
    log(f"case e4m3 sparse ps={ps} heads={hq},{hkv}")
    lens = [1, 0, 17, 100, 700, 1500, 2000, 16 * ps]
    c = Case(ps, lens, hq, hkv, ps)
    c.poison()
    for counts in ([1] * 8, [1, 3, 2, 3, 5, 7, 9, 16], [100] * 8):
        idx = c.lists(counts, 130)
        k = [min(n, max(0, -(-L // ps))) for n, L in zip(counts, lens)]
        for dt in (S.SPARROW_OUT_F32, S.SPARROW_OUT_BF16):
            c.check(sparse(c, k, idx, out_dtype=dt), c.formula(idx, k), (ps, counts, dt))


def test_sparse_odd_lists():
    # unsorted, repeated, out-of-range and empty lists; budgets above the row and below zero
    c = Case(9, [500, 500, 500, 500, 37], 8, 2, 16, absent=[(2, 4, -1)])
    c.poison()
    idx = c.lists([20, 20, 20, 20, 3], 24, sort=False)
    idx[0, 0, 3] = idx[0, 0, 4] = idx[0, 0, 5]       # the same page three times
    idx[1, 1, 0] = 1 << 30
    idx[1, 1, 1] = -9
    idx[1, 0, :] = -1                                # nothing at all
    idx[2, :, 0] = 4
    k = [20, 20, 20, 99, -2]
    c.check(sparse(c, k, idx), c.formula(idx, k), "odd lists")


@pytest.mark.parametrize("spread", [8, 30])
def test_rows_of_different_sizes(spread):
    # (q small enough that the logits stay within a few hundred)
    c = Case(spread, [333, 1000, 7], 8, 2, 32, spread=spread)
    c.q *= 2.0 ** -spread
    c.poison()
    c.check(dense(c), c.formula(), "spread")
    # zero rows among them: their exponent is the least, their weight counts
    c.k8.view(torch.uint8)[:, :, ::3] = 0
    c.v8.view(torch.uint8)[:, :, 1::3] = 0
    for j in (0, 1):
        e = c.exps[:, :, :, j].reshape(c.kv.shape[:3])
        e[:, :, j::3] = 10
        c.exps[:, :, :, j] = e.view(c.kv.shape[0], 2, -1, 4)
    c.kv[:, :, ::3] = 0
    c.vv[:, :, 1::3] = 0
    c.check(dense(c), c.formula(), "zero rows")


@pytest.mark.parametrize("scale", [0.0, -0.05, 1.0])
def test_scales(scale):
    c = Case(4, [70, 515], 12, 3, 16)
    c.check(dense(c, scale=scale), c.formula(scale=scale), scale)


def test_offsets_past_32_bits():
    # pages at the far end of caches of 5 GiB each
    hkv, ps, P = 8, 32, 163840
    k8, v8, exps = S.new_cache_e4m3(P, hkv, ps, DEV)
    c = Case(11, [150, 31], 16, hkv, ps)
    n = c.k8.shape[0]
    for big, small in ((k8, c.k8), (v8, c.v8), (exps, c.exps)):
        big.view(torch.uint8)[P - n:] = small.view(torch.uint8)
    want = c.formula()
    bt = torch.where(c.bt >= 0, c.bt + (P - n), c.bt)
    got = S.dense_decode_attn_e4m3(c.q, k8, v8, exps, bt, c.seq_lens)
    c.check(got, want, "far pages")
    # and the rows written and read there
    meta = S.new_meta(P, hkv, DEV)
    g = torch.Generator().manual_seed(1)
    rows = torch.randn((2, hkv, D), generator=g).to(torch.bfloat16).to(DEV)
    S.append_kv_e4m3(rows, rows, k8, v8, exps, bt, c.seq_lens, meta)
    ko, vo = S.read_kv_e4m3(k8, v8, exps, bt, c.seq_lens, None, 2)
    y, e = e4m3.quantise(rows.float().cpu().numpy())
    np.testing.assert_array_equal(ko.float().cpu().numpy(), np.ldexp(y, e[..., None]))
    assert torch.equal(ko, vo)


def test_against_the_bf16_attention_of_the_same_values():
    # the bf16 library call on a cache that holds the e4m3 cache's values (its numerators have 8 bits:
    # 2^-8 of sum w |v|, against the same tolerance as above)
    c = Case(12, [900, 20, 333], 16, 4, 16)
    kb, vb = (torch.from_numpy(x).to(torch.bfloat16).to(DEV) for x in (c.kv, c.vv))
    a = S.dense_decode_attn(c.q, kb, vb, c.bt, c.seq_lens)
    b = dense(c)
    _, size, far = c.formula()
    tol = (2.0 ** -15 * far[..., None] + 2.0 ** -13 + 2.0 ** -7) * size
    assert (np.abs((a - b).cpu().numpy()) <= tol).all()


def test_repeated_calls_graphs_and_streams():
    c = Case(13, [3000, 17, 0, 1200], 16, 4, 16)
    idx = c.lists([60, 2, 0, 40], 64)
    kt, it = torch.tensor([60, 2, 0, 40], dtype=torch.int32, device=DEV), torch.from_numpy(idx).to(DEV)
    args = (c.q, c.k8, c.v8, c.exps, c.bt, c.seq_lens)
    want = dense(c), S.sparse_decode_attn_e4m3(*args, kt, it)
    assert torch.equal(dense(c), want[0])
    shape = S.make_shape(4, 16, 4, 16, c.bt.shape[1], c.k8.shape[0])
    ws = [torch.empty(S.sparrow_workspace_size(shape, 64, op), dtype=torch.uint8, device=DEV)
          for op in (S.SPARROW_OP_DENSE_ATTN, S.SPARROW_OP_SPARSE_ATTN)]
    outs = [torch.empty_like(w) for w in want]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert torch.equal(dense(c), want[0])
        with torch.cuda.graph(graph, stream=side):
            S.dense_decode_attn_e4m3(*args, out=outs[0], workspace=ws[0])
            S.sparse_decode_attn_e4m3(*args, kt, it, out=outs[1], workspace=ws[1])
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(3):
        for t in outs + ws:
            t.view(torch.uint8).fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1]), rep


def test_wrapper_refusals():
    c = Case(14, [30, 40], 4, 2, 16)
    ok = dict(q=c.q, k_cache=c.k8, v_cache=c.v8, exps=c.exps, block_table=c.bt, seq_lens=c.seq_lens)
    idx = torch.zeros((2, 2, 3), dtype=torch.int32, device=DEV)
    k = torch.ones(2, dtype=torch.int32, device=DEV)
    small = torch.empty(64, dtype=torch.uint8, device=DEV)
    for kw in (dict(q=c.q.float()), dict(q=c.q[:1]), dict(q=c.q[:, :3]), dict(q=c.q[..., :64]),
               dict(k_cache=c.k8.view(torch.uint8)), dict(v_cache=c.v8[1:]), dict(exps=c.exps[:, :1]),
               dict(block_table=c.bt.long()), dict(seq_lens=c.seq_lens[:1]),
               dict(workspace=small), dict(out=torch.empty(2, 4, D, dtype=torch.bfloat16, device=DEV)),
               dict(out_dtype=7), dict(block_table=c.bt.t())):
        with pytest.raises((ValueError, RuntimeError)):
            S.dense_decode_attn_e4m3(**(ok | kw))
        with pytest.raises((ValueError, RuntimeError)):
            S.sparse_decode_attn_e4m3(**(ok | kw), k=k, idx=idx)
    for kw in (dict(k=k.long()), dict(k=k[:1]), dict(idx=idx[:, :1]), dict(idx=idx.long()),
               dict(idx=idx[:, :, 0])):
        with pytest.raises(ValueError):
            S.sparse_decode_attn_e4m3(**ok, **(dict(k=k, idx=idx) | kw))


def test_the_steps_together():
    # two decode steps behind a prompt, as a program runs them: projections in one buffer, norms and
    # rotation, the cache, page selection by its landmarks, attention; each stage against 64 bits
    # on what the stage before gave
    B, hq, hkv, ps, eps = 3, 8, 2, 16, 1e-6
    g = torch.Generator().manual_seed(15)
    prompt = [180, 1, 77]
    pages = [n // ps + 2 for n in prompt]
    P = sum(pages)
    perm, at = torch.randperm(P, generator=g).to(torch.int32), 0
    bt = torch.zeros((B, max(pages)), dtype=torch.int32)
    for b, n in enumerate(pages):
        bt[b, :n] = perm[at:at + n]
        at += n
    bt = bt.to(DEV)
    k8, v8, exps = S.new_cache_e4m3(P, hkv, ps, DEV)
    meta = S.new_meta(P, hkv, DEV)
    wq, wk = ((1 + 0.2 * torch.randn(D, generator=g)).to(torch.bfloat16).to(DEV) for _ in range(2))
    freq = torch.from_numpy(1e6 ** (-np.arange(0, D, 2) / D)).to(DEV)
    table = torch.tensor([3], dtype=torch.int32, device=DEV)
    zero = torch.zeros(1, dtype=torch.int32, device=DEV)
    lens = np.zeros(B, np.int64)
    for step in range(3):
        new = prompt if step == 0 else [1] * B
        lens = lens + new
        T = sum(new)
        cu = None if step else torch.tensor(np.concatenate([[0], np.cumsum(new)]),
                                            dtype=torch.int32, device=DEV)
        pos = torch.tensor(np.concatenate([np.arange(L - n, L) for L, n in zip(lens, new)]),
                           dtype=torch.int32, device=DEV)
        seq_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        qkv = torch.randn((T, (hq + 2 * hkv) * D), generator=g).to(torch.bfloat16).to(DEV)
        q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([hq * D, hkv * D, hkv * D], 1))
        q, k = S.qk_norm_rope(q, k, wq, wk, freq, pos, eps)
        S.append_kv_e4m3(k, v, k8, v8, exps, bt, seq_lens, meta, cu_tokens=cu)
        if step == 0:
            continue
        kv, vv = e4m3.both_values(k8, v8, exps)
        for b in range(B):          # the new rows are in the cache
            y, e = e4m3.quantise(k[b].float().cpu().numpy())
            pg, sl = divmod(int(lens[b]) - 1, ps)
            np.testing.assert_array_equal(kv[int(bt[b, pg]), :, sl], np.ldexp(y, e[:, None]))
        cache = torch.from_numpy(kv).to(torch.bfloat16).to(DEV)
        rebuilt = torch.zeros_like(meta)
        S.page_meta_update(cache, bt, seq_lens, rebuilt)
        used = torch.cat([bt[b, :-(-int(L) // ps)] for b, L in enumerate(lens)]).long()
        assert torch.equal(meta[used], rebuilt[used])
        kk, idx = S.page_score_topk(q, meta, bt, seq_lens, (P, hkv, ps, D), table, zero, 1, 2048, 4)
        out = S.sparse_decode_attn_e4m3(q, k8, v8, exps, bt, seq_lens, kk, idx)
        c = Case.__new__(Case)
        c.hq, c.hkv, c.ps, c.lens, c.q, c.kv, c.vv = hq, hkv, ps, lens, q, kv, vv
        c.bt_host = bt.cpu().numpy()
        c.check(out, c.formula(idx.cpu().numpy(), kk.cpu().numpy()), f"step {step}")
        assert kk.tolist() == [3, 1, 3]


def test_workload_shapes_have_landmarks_that_bound_the_stored_keys():
    # an upper bound of q . k over a page, of the values as stored: min/max landmarks of an e4m3 cache
    w = W.small(B=2, Hq=8, Hkv=2, ps=16, lengths=(100, 61), seed=3)
    inp = W.generate(w, DEV, lengths=[100, 61])
    P = inp.k_cache.shape[0]
    k8, v8, exps = S.new_cache_e4m3(P, 2, 16, DEV)
    meta = S.new_meta(P, 2, DEV)
    rows = torch.cat([inp.k_cache[inp.block_table[b].long()].transpose(1, 2).reshape(-1, 2, D)[:L]
                      for b, L in enumerate((100, 61))]).contiguous()
    S.append_kv_e4m3(rows, rows, k8, v8, exps, inp.block_table, inp.seq_lens, meta,
                     cu_tokens=torch.tensor([0, 100, 161], dtype=torch.int32, device=DEV))
    kv, _ = e4m3.both_values(k8, v8, exps)
    m = meta.float().cpu().numpy()
    for b, L in enumerate((100, 61)):
        for pos in range(L):
            ph = int(inp.block_table[b, pos // 16])
            assert (m[ph, :, 0] <= kv[ph, :, pos % 16]).all()
            assert (m[ph, :, 1] >= kv[ph, :, pos % 16]).all()


@pytest.mark.parametrize("B", [4097, 8000])
def test_very_many_short_sequences(B):
    # the search over the page offsets takes three rounds; empty sequences among them
    log(f"case e4m3 attention very many sequences B={B}")
    g = np.random.default_rng(B)
    c = Case(B, (g.integers(0, 30, B) * (g.random(B) < 0.7)).tolist(), 2, 1, 16)
    c.poison()
    c.check(dense(c), c.formula(), "dense")
    counts = g.integers(-1, 3, B).tolist()
    idx = c.lists([max(0, n) for n in counts], 2)
    c.check(sparse(c, counts, idx), c.formula(idx, counts), "sparse")


def test_calls_at_once_on_two_streams():
    # both kernels, each stream with its own workspaces and outputs
    cases = [Case(40 + i, [4000 - 900 * i, 17, 300], 8, 2, 16) for i in range(2)]
    lists = [c.lists([12, 2, 9], 16) for c in cases]
    want = [(dense(c), sparse(c, [12, 2, 9], i)) for c, i in zip(cases, lists)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for rep in range(8):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                got[i].append((dense(c), sparse(c, [12, 2, 9], lists[i])))
    torch.cuda.synchronize()
    for outs, w in zip(got, want):
        assert all(torch.equal(o, x) for pair in outs for o, x in zip(pair, w))


# both sides of the sizes up to which a (sequence, KV head) is one workgroup's (256 CUs)
@pytest.mark.parametrize("B,hkv,ps,k_max", [(96, 8, 16, 64), (97, 8, 16, 5), (32, 8, 32, 64), (33, 8, 32, 64),
                                            (16, 8, 64, 32), (17, 8, 128, 16), (3, 8, 64, 17)])
def test_sparse_sizes_around_the_split(B, hkv, ps, k_max):
    log(f"case e4m3 split B={B} ps={ps} k_max={k_max}")
    g = np.random.default_rng(B + ps)
    lens = g.integers(1, 2 * ps * k_max // 3 + 2, B)
    lens[:3] = [0, 1, ps * k_max + 5]
    c = Case(B, lens[:B].tolist(), 2 * hkv, hkv, ps)
    c.poison()
    counts = g.integers(0, k_max + 1, B).tolist()
    counts[B - 1] = k_max + 3
    idx = c.lists([min(n, k_max) for n in counts], k_max)
    c.check(sparse(c, counts, idx), c.formula(idx, counts), "split")
