"""Writing and reading an e4m3 cache against the format's definition in 64 bits (tests/e4m3.py):
codes, exponents, landmarks and rows are exact."""
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


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Cache:
    """A cache with random contents, its block table, and a plain copy of both."""

    def __init__(self, seed, hkv, ps, lens, mean=False, spare=2):
        g = torch.Generator().manual_seed(seed)
        self.g, self.hkv, self.ps, self.mean = g, hkv, ps, mean
        pages = [max(0, -(-int(L) // ps)) + 1 for L in lens]
        P = sum(pages) + spare
        perm = torch.randperm(P, generator=g).numpy()
        bt = np.full((len(lens), max(pages)), -1, np.int32)
        at = 0
        for b, n in enumerate(pages):
            bt[b, :n] = perm[at:at + n]
            at += n
        self.lens_host, self.bt_host = np.array(lens, np.int32), bt
        self.k8, self.v8, self.exps = S.new_cache_e4m3(P, hkv, ps, DEV)
        self.meta = S.new_meta(P, hkv, DEV, S.SPARROW_LANDMARK_MEAN if mean else 0)
        for c in (self.k8, self.v8):
            c.copy_(torch.randn(c.shape, generator=g).clamp(-400, 400).to(DEV))
        self.exps.copy_(torch.randint(100, 140, self.exps.shape, generator=g).to(DEV))
        self.meta.copy_(torch.randn(self.meta.shape, generator=g).to(DEV))
        self.upload()

    def upload(self):
        self.bt = torch.from_numpy(self.bt_host).to(DEV)
        self.lens = torch.from_numpy(self.lens_host).to(DEV)

    def rows(self, T, scale=1.0):
        """K contiguous, V inside a fused projection's rows."""
        k = (torch.randn((T, self.hkv, D), generator=self.g) * scale).to(torch.bfloat16).to(DEV)
        v = torch.randn((T, 3 * self.hkv * D), generator=self.g).to(torch.bfloat16).to(DEV)
        return k, v[:, 2 * self.hkv * D:].unflatten(1, (self.hkv, D))

    def append_and_check(self, k, v, cu):
        kv, vv = e4m3.both_values(self.k8, self.v8, self.exps)
        meta = f64(self.meta)
        landmark = S.SPARROW_LANDMARK_MEAN if self.mean else 0
        S.append_kv_e4m3(k, v, self.k8, self.v8, self.exps, self.bt, self.lens, self.meta,
                         cu_tokens=None if cu is None else torch.tensor(cu, dtype=torch.int32,
                                                                        device=DEV),
                         landmark=landmark)
        cu = list(range(len(self.lens_host) + 1)) if cu is None else cu
        e4m3.append(f64(k), f64(v), cu, self.bt_host, self.lens_host, self.ps, kv, vv, meta,
                    self.mean)
        got = e4m3.both_values(self.k8, self.v8, self.exps)
        np.testing.assert_array_equal(got[0], kv)
        np.testing.assert_array_equal(got[1], vv)
        np.testing.assert_array_equal(f64(self.meta), meta)


def test_every_bf16_pattern():
    # all finite patterns, as rows around one magnitude and as rows of mixed magnitudes
    bits = np.arange(65536, dtype=np.uint16)
    bits = bits[(bits & 0x7f80) != 0x7f80]
    g = np.random.default_rng(0)
    both = np.concatenate([bits, g.permutation(bits)])
    T = len(both) // D
    x = torch.from_numpy(both[:T * D].astype(np.int16)).view(torch.bfloat16).view(T, 1, D).to(DEV)
    k8, v8, exps = S.new_cache_e4m3(T, 1, 16, DEV)
    bt = torch.arange(T, dtype=torch.int32, device=DEV).view(T, 1)
    lens = torch.ones(T, dtype=torch.int32, device=DEV)
    meta = S.new_meta(T, 1, DEV)
    S.append_kv_e4m3(x, x, k8, v8, exps, bt, lens, meta)
    y, e = e4m3.quantise(f64(x))
    np.testing.assert_array_equal(f64(k8)[:, :, 0], y)
    np.testing.assert_array_equal(f64(v8)[:, :, 0], y)
    np.testing.assert_array_equal(exps[:, :, 0, 0, 0].cpu().numpy(), e + 127)
    np.testing.assert_array_equal(exps[:, :, 0, 1, 0].cpu().numpy(), e + 127)
    ko, vo = S.read_kv_e4m3(k8, v8, exps, bt, lens, None, T)
    np.testing.assert_array_equal(f64(ko), np.ldexp(y, e[..., None]))     # exact in bf16
    assert torch.equal(ko, vo)
    np.testing.assert_array_equal(f64(meta)[:, :, 0], f64(ko))
    # the sign of a zero stays
    assert torch.equal(torch.signbit(ko), torch.signbit(x))
    # the same rows through the page writer
    k2, v2, e2 = S.new_cache_e4m3(T, 1, 16, DEV)
    m2 = S.new_meta(T, 1, DEV)
    S.append_kv_e4m3(x, x, k2, v2, e2, bt, lens, m2,
                     cu_tokens=torch.arange(T + 1, dtype=torch.int32, device=DEV))
    for a, b in ((k8, k2), (v8, v2), (exps, e2)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(meta.view(torch.int16), m2.view(torch.int16))


def test_infinities_become_the_largest_value():
    k8, v8, exps = S.new_cache_e4m3(2, 1, 16, DEV)
    x = torch.zeros((1, 1, D), dtype=torch.bfloat16, device=DEV)
    x[0, 0, 3], x[0, 0, 4], x[0, 0, 5] = float("inf"), float("-inf"), 2.0 ** 120
    one = torch.ones(1, dtype=torch.int32, device=DEV)
    bt = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    S.append_kv_e4m3(x, x, k8, v8, exps, bt, one, S.new_meta(2, 1, DEV))
    ko, _ = S.read_kv_e4m3(k8, v8, exps, bt, one, None, 1)
    top = 448 * 2.0 ** 119
    assert ko[0, 0, 3:6].tolist() == [top, -top, 2.0 ** 120]


@pytest.mark.parametrize("ps", [16, 32, 64, 128])
@pytest.mark.parametrize("mean", [False, True])
def test_decode_append(ps, mean):
    log(f"case e4m3 decode append ps={ps} mean={mean}")
    lens = [1, ps, ps + 1, 5 * ps - 3, 0, 2, -4, 700]
    c = Cache(ps, 3, ps, lens, mean)
    c.bt_host[5, 0] = 1 << 30                    # an absent page
    c.lens_host[7] = c.bt_host.shape[1] * ps + 1    # beyond its table
    c.upload()
    k, v = c.rows(len(lens), scale=3.0)
    c.append_and_check(k, v, None)


@pytest.mark.parametrize("ps", [16, 32, 64, 128])
@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("hkv", [1, 3, 8])
def test_prompt_append(ps, mean, hkv):
    log(f"case e4m3 prompt append ps={ps} mean={mean} hkv={hkv}")
    new = [1, 0, ps, 3 * ps + 5, 17, 2 * ps, 7, 200]
    past = [0, 9, 0, 3, ps - 1, 2 * ps, ps - 7, 133]
    lens = [n + p for n, p in zip(new, past)]
    c = Cache(31 + ps, hkv, ps, lens, mean)
    cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    k, v = c.rows(cu[-1] + 5)                    # five rows behind the last sequence
    k[cu[-1]:] = float("nan")
    c.append_and_check(k, v, cu)


def test_prompt_append_edges():
    # longer than its length, empty and negative lengths, absent pages, rows past the block table
    ps = 16
    c = Cache(7, 2, ps, [40, 3, 0, 33, 50, 20])
    c.bt_host[3, 1] = -1
    c.bt_host[4, 2] = 1 << 20
    c.lens_host[:] = [40, 3, 0, 33, 50, -7]
    c.upload()
    new = [40, 20, 8, 33, 21, 5]
    cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    k, v = c.rows(cu[-1])
    c.append_and_check(k, v, cu)
    c.lens_host[0] = c.bt_host.shape[1] * ps + 1
    c.upload()
    c.append_and_check(k, v, cu)


def test_row_offsets_outside_the_rows_stay_inside():
    c = Cache(8, 2, 16, [64, 64, 64])
    k, v = c.rows(30)
    before = [t.clone() for t in (c.k8, c.v8, c.exps, c.meta)]
    cu = torch.tensor([-5, 1 << 30, 1 << 30, 1 << 30], dtype=torch.int32, device=DEV)
    S.append_kv_e4m3(k, v, c.k8, c.v8, c.exps, c.bt, c.lens, c.meta, cu_tokens=cu)
    # the first sequence has all 30 rows, the others none
    want = Cache(8, 2, 16, [64, 64, 64])
    want.append_and_check(k, v, [0, 30, 30, 30])
    for a, b in zip((c.k8, c.v8, c.exps), (want.k8, want.v8, want.exps)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert not torch.equal(before[0].view(torch.uint8), c.k8.view(torch.uint8))


@pytest.mark.parametrize("B", [1, 65, 300])
def test_many_short_prompts(B):
    # the search over the row offsets takes one and two trips
    g = np.random.default_rng(B)
    new = g.integers(0, 9, B)
    past = g.integers(0, 40, B)
    c = Cache(B, 2, 16, (new + past).tolist())
    cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    k, v = c.rows(max(1, cu[-1]))
    c.append_and_check(k, v, cu)


def test_token_by_token_equals_one_prompt():
    for mean in (False, True):
        a, b = (Cache(3, 4, 32, [71, 33], mean) for _ in range(2))
        k, v = a.rows(104)
        a.append_and_check(k, v, [0, 71, 104])
        for t in range(71):
            b.lens_host[:] = [t + 1, max(0, t - 37)]
            b.upload()
            rows = torch.tensor([t, 71 + max(0, t - 38)], device=DEV)
            b.append_and_check(k[rows], v[rows], None)
        b.lens_host[:] = [0, 33]
        assert torch.equal(a.k8.view(torch.uint8), b.k8.view(torch.uint8))
        assert torch.equal(a.exps, b.exps)
        assert torch.equal(a.meta, b.meta)


def test_landmarks_equal_a_rebuild_of_the_values():
    # page_meta_update over a bf16 cache that holds what the 8-bit one stands for
    for mean in (False, True):
        lm = S.SPARROW_LANDMARK_MEAN if mean else 0
        c = Cache(4, 2, 16, [100, 37], mean)
        k, v = c.rows(137)
        c.append_and_check(k, v, [0, 100, 137])
        kv, _ = e4m3.both_values(c.k8, c.v8, c.exps)
        cache = torch.from_numpy(kv).to(torch.bfloat16).to(DEV)
        meta = c.meta.clone()
        S.page_meta_update(cache, c.bt, c.lens, meta, landmark=lm)
        assert torch.equal(meta, c.meta)


@pytest.mark.parametrize("ps", [16, 32, 64, 128])
def test_read(ps):
    log(f"case e4m3 read ps={ps}")
    lens = [1, 5 * ps + 3, 0, 2 * ps, 300, 9, 77]
    c = Cache(50 + ps, 3, ps, lens)
    c.bt_host[4, 1] = -3
    c.lens_host[6] = c.bt_host.shape[1] * ps + 20       # past its block table
    c.upload()
    new = [1, 2 * ps + 7, 0, 2 * ps, 300, 12, 60]       # one goes before position 0
    cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    T = cu[-1] + 4
    ko = torch.full((T, 3, D), 5.0, dtype=torch.bfloat16, device=DEV)
    vo = ko.clone()
    S.read_kv_e4m3(c.k8, c.v8, c.exps, c.bt, c.lens,
                   torch.tensor(cu, dtype=torch.int32, device=DEV), T, k_out=ko, v_out=vo)
    kv, vv = e4m3.both_values(c.k8, c.v8, c.exps)
    np.testing.assert_array_equal(f64(ko), e4m3.read(kv, cu, c.bt_host, c.lens_host, T, 5.0))
    np.testing.assert_array_equal(f64(vo), e4m3.read(vv, cu, c.bt_host, c.lens_host, T, 5.0))
    # without offsets: the last token of each
    ko, vo = S.read_kv_e4m3(c.k8, c.v8, c.exps, c.bt, c.lens, None, len(lens))
    one = list(range(len(lens) + 1))
    np.testing.assert_array_equal(f64(ko), e4m3.read(kv, one, c.bt_host, c.lens_host, len(lens), 0))


def test_wrapper_refusals():
    c = Cache(1, 2, 16, [20, 30])
    k, v = c.rows(9)
    cu = torch.tensor([0, 4, 9], dtype=torch.int32, device=DEV)

    def write(**kw):
        a = dict(k_new=k, v_new=v, k_cache=c.k8, v_cache=c.v8, exps=c.exps, block_table=c.bt,
                 seq_lens=c.lens, meta=c.meta, cu_tokens=cu) | kw
        S.append_kv_e4m3(**a)
    for kw in (dict(k_new=k.float()), dict(k_new=k[:8]), dict(k_new=k[..., :64]), dict(cu_tokens=None),
               dict(cu_tokens=cu[:2]), dict(cu_tokens=cu.long()), dict(exps=c.exps[:1]),
               dict(exps=c.exps.int()), dict(k_cache=c.k8.view(torch.uint8)), dict(v_cache=c.v8[:3]),
               dict(seq_lens=c.lens.long()), dict(meta=c.meta.float()), dict(block_table=c.bt.long()),
               dict(landmark=S.SPARROW_LANDMARK_MEAN), dict(v_new=v.transpose(0, 1))):
        with pytest.raises((ValueError, RuntimeError)):
            write(**kw)
    with pytest.raises(ValueError):
        S.read_kv_e4m3(c.k8, c.v8, c.exps, c.bt, c.lens, cu, 9,
                       k_out=torch.empty(8, 2, D, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(S.SparrowError):
        S.read_kv_e4m3(c.k8, c.v8, c.exps, c.bt, c.lens, None, 5)     # two sequences
    with pytest.raises(ValueError):
        S.read_kv_e4m3(c.k8, c.v8, c.exps, c.bt, c.lens, cu, -1, k_out=k[:0], v_out=k[:0])


def test_graph_replays_and_side_stream():
    c, want = (Cache(2, 4, 16, [90, 33, 200]) for _ in range(2))
    k, v = c.rows(323)
    cu = torch.tensor([0, 90, 123, 323], dtype=torch.int32, device=DEV)
    want.append_and_check(k, v, [0, 90, 123, 323])
    ref = S.read_kv_e4m3(want.k8, want.v8, want.exps, want.bt, want.lens, cu, 323)
    empty = [t.clone() for t in (c.k8, c.v8, c.exps, c.meta)]
    ko, vo = (torch.zeros_like(r) for r in ref)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        S.append_kv_e4m3(k, v, c.k8, c.v8, c.exps, c.bt, c.lens, c.meta, cu_tokens=cu)
        S.read_kv_e4m3(c.k8, c.v8, c.exps, c.bt, c.lens, cu, 323, k_out=ko, v_out=vo)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(3):
        for t, e in zip((c.k8, c.v8, c.exps, c.meta), empty):
            t.view(torch.uint8).copy_(e.view(torch.uint8))
        ko.zero_()
        vo.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ko, ref[0]) and torch.equal(vo, ref[1]), rep
        assert torch.equal(c.meta, want.meta) and torch.equal(c.exps, want.exps), rep
        assert torch.equal(c.k8.view(torch.uint8), want.k8.view(torch.uint8)), rep


def test_bf16_bits_of_landmarks_keep_their_zero_signs():
    # -0 orders below +0, as in the landmark build
    c = Cache(6, 1, 16, [3])
    k = torch.zeros((3, 1, D), dtype=torch.bfloat16, device=DEV)
    k[1] = -0.0
    S.append_kv_e4m3(k, k, c.k8, c.v8, c.exps, c.bt, c.lens, c.meta,
                     cu_tokens=torch.tensor([0, 3], dtype=torch.int32, device=DEV))
    m = W.bf16_bits(c.meta[c.bt[0, 0].long()])
    assert (m[0, 0] == 0x8000).all() and (m[0, 1] == 0).all()


def test_very_many_sequences():
    # the search over the row offsets takes three trips; decode rows as well
    B = 4097
    g = np.random.default_rng(B)
    new = g.integers(0, 4, B)
    past = g.integers(0, 20, B)
    c = Cache(B, 1, 16, (new + past).tolist())
    cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    k, v = c.rows(max(1, cu[-1]))
    c.append_and_check(k, v, cu)
    k, v = c.rows(B)
    c.append_and_check(k, v, None)
    ko, _ = S.read_kv_e4m3(c.k8, c.v8, c.exps, c.bt, c.lens, None, B)
    kv, _ = e4m3.both_values(c.k8, c.v8, c.exps)
    np.testing.assert_array_equal(
        f64(ko), e4m3.read(kv, list(range(B + 1)), c.bt_host, c.lens_host, B, 0))


def test_row_offsets_past_32_bits():
    # 2.4e9 elements of new rows and of rows read back, from two sequences
    hkv, ps, n = 8, 128, 300
    lens = [1200000, 1100003]
    T = sum(lens)
    pages = [-(-L // ps) for L in lens]
    k8, v8, exps = S.new_cache_e4m3(sum(pages), hkv, ps, DEV)
    meta = S.new_meta(sum(pages), hkv, DEV)
    bt = torch.full((2, max(pages)), -1, dtype=torch.int32, device=DEV)
    bt[0, :pages[0]] = torch.arange(pages[0], device=DEV, dtype=torch.int32)
    bt[1, :pages[1]] = torch.arange(pages[0], sum(pages), device=DEV, dtype=torch.int32)
    seq_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    cu = torch.tensor([0, lens[0], T], dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(32)
    rows = torch.randn((T, hkv, D), generator=g, device=DEV, dtype=torch.bfloat16)
    S.append_kv_e4m3(rows, rows, k8, v8, exps, bt, seq_lens, meta, cu_tokens=cu)
    ko, vo = S.read_kv_e4m3(k8, v8, exps, bt, seq_lens, cu, T)
    for at in (slice(T - n, T), slice(lens[0] - n, lens[0] + n), slice(0, n)):
        y, e = e4m3.quantise(f64(rows[at]))
        np.testing.assert_array_equal(f64(ko[at]), np.ldexp(y, e[..., None]))
        assert torch.equal(ko[at], vo[at])
