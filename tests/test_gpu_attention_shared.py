"""Decode attention of groups with a shared prefix against the formula in 64 bits (on the CPU).

Tolerances.  With S = sum_t w_t |V[t]| (per channel) and Z = scale sum_i |q_i K[t]_i| (at most, over the
tokens): a logit is 128 products in four chains of matrix instructions and one factor, off by 2^-17.5 of Z
at most (128 + 4 roundings of 2^-24), and moves its weight by that much; the exponential, the sums over
a wave's tiles (under 600 here), the waves' parts and the division add 2^-14.  fp32 output: (2 * 2^-17.5 Z +
2^-14) S, the 2 for numerator and denominator.  bf16 output: the numerators' rounding, 2^-8 each on
weights and sum at most, and the output's own: (2^-7 + ...) S + 2^-8 |out|.  They are bounds: the
errors' mean is far below, and is bounded too, at a tenth."""
import math

import numpy as np
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
D = 128
F32, BF16 = S.SPARROW_OUT_F32, S.SPARROW_OUT_BF16


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


class Case:
    """Groups of `per` sequences with prefixes `pre`; sequence lengths `lens`.  Rows of the block table
    hold the group's pages first; entries that are not to be read name a page of NaN."""

    def __init__(self, per, pre, lens, hq=8, hkv=2, ps=16, seed=0, extra=0, nan=True, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.per, self.pre, self.ps, self.hkv, self.hq = per, pre, ps, hkv, hq
        self.lens = [int(x) for x in lens]
        B = len(self.lens)
        M = max([1] + [-(-n // ps) for n in self.lens] + [p // ps for p in pre]) + extra
        need = [-(-n // ps) for n in self.lens]
        P = sum(need) + sum(p // ps for p in pre) + 1 + spare
        perm = torch.randperm(P, generator=g).tolist()
        trap = perm.pop()
        bt = np.full((B, M), trap, np.int64)
        self.full = np.full((B, M), trap, np.int64)     # the pages that each sequence's tokens lie on
        self.cu = [0]
        b = 0
        for n, p in zip(per, pre):
            s = min(p // ps, M) if n > 1 else 0
            shared = [perm.pop() for _ in range(s)]
            for i in range(n):
                if i == 0:
                    bt[b, :s] = shared
                own = [perm.pop() for _ in range(max(0, need[b] - s))]
                bt[b, s:s + len(own)] = own
                self.full[b, :s] = shared
                self.full[b, s:s + len(own)] = own
                b += 1
            self.cu.append(b)
        for b in range(b, B):                           # in no group
            own = [perm.pop() for _ in range(need[b])]
            bt[b, :len(own)] = self.full[b, :len(own)] = own
        self.k = torch.randn((P, hkv, ps, D), generator=g).to(torch.bfloat16)
        self.v = torch.randn((P, hkv, ps, D), generator=g).to(torch.bfloat16)
        self.q = torch.randn((B, hq, D), generator=g).to(torch.bfloat16)
        if nan:                                         # whatever no sequence's tokens are on
            used = torch.zeros((P, ps), dtype=torch.bool)
            for b, n in enumerate(self.lens):
                for t in range(n):
                    used[self.full[b, t // ps], t % ps] = True
            for c in (self.k, self.v):
                c[~used[:, None].expand(P, hkv, ps)] = math.nan
        self.bt = torch.from_numpy(bt.astype(np.int32)).to(DEV)

    def args(self):
        i32 = dict(dtype=torch.int32, device=DEV)
        return (self.q.to(DEV), self.k.to(DEV), self.v.to(DEV), self.bt,
                torch.tensor(self.lens, **i32), torch.tensor(self.cu, **i32),
                torch.tensor(self.pre, **i32))

    def reference(self, scale):
        """(out, S, largest Z of the row) in 64 bits."""
        B, G, ps = len(self.lens), self.hq // self.hkv, self.ps
        out = torch.zeros((B, self.hq, D), dtype=torch.float64)
        size, most = torch.zeros_like(out), torch.zeros((B, self.hq, 1), dtype=torch.float64)
        P = self.k.shape[0]
        for b, n in enumerate(self.lens):
            at = torch.arange(n)
            page = torch.from_numpy(self.full[b])[at // ps]
            ok = (page >= 0) & (page < P)
            at, page = at[ok], page[ok]
            if len(at) == 0:
                continue
            for h in range(self.hkv):
                k, v = self.k[page, h, at % ps].double(), self.v[page, h, at % ps].double()
                q = self.q[b, h * G:(h + 1) * G].double()
                z = scale * q @ k.T
                w = torch.softmax(z, -1)
                rows = slice(h * G, (h + 1) * G)
                out[b, rows] = w @ v
                size[b, rows] = w @ v.abs()
                most[b, rows] = abs(scale) * (q.abs() @ k.abs().T).amax(-1, keepdim=True)
        return out, size, most

    def check(self, dtype=F32, scale=1 / math.sqrt(D), got=None):
        if got is None:
            got = S.shared_prefix_decode_attn(*self.args(), scale=scale, out_dtype=dtype)
        want, size, most = self.reference(scale)
        err = (got.cpu().double() - want).abs()
        tol = (2 * 2 ** -17.5 * most + 2 ** -14) * size + 1e-30
        if dtype == BF16:
            tol = tol + 2 ** -7 * size + 2 ** -8 * want.abs()
        assert got.dtype == (torch.float32 if dtype == F32 else torch.bfloat16)
        assert bool((err <= tol).all()), float((err - tol).max())
        assert float(err.mean()) <= 0.1 * float(tol.mean()) + 1e-30
        return got


def rng_lens(seed, per, pre, lo, hi):
    r = np.random.default_rng(seed)
    return [p + int(x) for n, p in zip(per, pre) for x in r.integers(lo, hi + 1, n)]


GROUPS = [([1], [40], 1, 1), ([2], [64], 1, 40), ([8], [500], 1, 64), ([3, 1, 5], [33, 200, 16], 1, 90),
          ([17, 2], [1, 1030], 1, 5), ([20], [15], 1, 300), ([1, 1, 1], [100, 7, 50], 1, 30),
          ([70], [130], 1, 9)]


@pytest.mark.parametrize("per,pre,lo,hi", GROUPS)
@pytest.mark.parametrize("hq,hkv,ps", [(2, 1, 16), (8, 2, 32), (10, 2, 64), (16, 1, 128), (3, 3, 16)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_groups(per, pre, lo, hi, hq, hkv, ps, dtype):
    log(f"case shared per={per} pre={pre} heads={hq},{hkv} ps={ps} out={dtype}")
    Case(per, pre, rng_lens(sum(per) + ps, per, pre, lo, hi), hq, hkv, ps, seed=sum(pre)).check(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_prefixes(dtype):
    log("case shared long")
    per, pre = [9, 4], [5000, 3333]
    Case(per, pre, rng_lens(1, per, pre, 1, 700), 8, 2, 16, seed=2, nan=False).check(dtype)
    Case([40], [9001], rng_lens(2, [40], [9001], 1, 100), 4, 1, 32, seed=3, nan=False).check(dtype)


def test_short_and_empty_sequences():
    # ended samples, sequences inside the shared part, a group with nothing at all
    for ps in (16, 64):
        per, pre = [5, 3, 2], [200, 100, 64]
        lens = [0, 250, 10, 200, 1, 0, 0, 0, 64, 3]
        c = Case(per, pre, lens, 8, 2, ps, seed=4)
        out = c.check()
        assert bool((out[[0, 5, 6, 7]] == 0).all())


def test_nobody_reaches_the_prefix_end():
    # prefix_lens beyond what any sequence has: tokens behind the longest may hold anything
    Case([3], [320], [100, 37, 64], 8, 2, 32, seed=5).check()


def test_sequences_outside_the_groups():
    c = Case([2, 2], [48, 20], [60, 70, 40, 33, 25, 90], 8, 2, 16, seed=6)
    c.check()
    # groups that begin behind the first sequence
    c = Case([1, 3], [99, 48], [60, 70, 80, 90, 30], 8, 2, 16, seed=7)
    want = c.check()
    a = list(c.args())
    a[5], a[6] = a[5][1:].contiguous(), a[6][1:].contiguous()
    # (sequence 0 is then in no group, which for a group of one changes nothing)
    out = S.shared_prefix_decode_attn(*a)
    c.check(got=out)
    assert out.shape == want.shape


def test_no_groups_equals_dense():
    c = Case([], [], [70, 0, 500, 33], 8, 2, 16, seed=8)
    c.check()
    c.check(BF16)
    a = c.args()
    c.check(got=S.dense_decode_attn(*a[:5], out_dtype=BF16), dtype=BF16)   # (the same tolerance)


def test_groups_out_of_range():
    # entries outside the batch count as the nearer end, falling ones as the one before
    c = Case([4], [64], [80, 90, 100, 70], 8, 2, 16, seed=9)
    want = S.shared_prefix_decode_attn(*c.args())
    a = list(c.args())
    a[5] = torch.tensor([-5, 9], dtype=torch.int32, device=DEV)
    assert torch.equal(S.shared_prefix_decode_attn(*a), want)
    a[5] = torch.tensor([0, 4, 2, -1, 7], dtype=torch.int32, device=DEV)
    a[6] = torch.tensor([64, 16, 1 << 30, -3], dtype=torch.int32, device=DEV)
    c.check(got=S.shared_prefix_decode_attn(*a))


def test_prefix_lens_out_of_range():
    # negative: nothing is shared (every row of the table is then read whole)
    c = Case([3], [64], [80, 90, 70], 8, 2, 16, seed=10, nan=False)
    a = list(c.args())
    a[3] = torch.from_numpy(c.full.astype(np.int32)).to(DEV)
    a[6] = torch.tensor([-64], dtype=torch.int32, device=DEV)
    c.check(got=S.shared_prefix_decode_attn(*a))
    # more than the table holds: everything is read from the first sequence's row
    c = Case([3], [96], [80, 96, 70], 8, 2, 16, seed=11)
    a = list(c.args())
    a[6] = torch.tensor([2 ** 31 - 1], dtype=torch.int32, device=DEV)
    c.check(got=S.shared_prefix_decode_attn(*a))


def test_absent_pages():
    for ps in (16, 32):
        c = Case([4], [6 * ps], [8 * ps, 7 * ps + 3, 6 * ps, 9 * ps], 8, 2, ps, seed=12)
        bad = c.bt.clone()
        bad[0, 1] = -1
        bad[0, 4] = c.k.shape[0]
        bad[1, 6] = 2 ** 31 - 1
        bad[3, 8] = -2 ** 31
        c.bt = bad
        c.full[:, 1] = c.full[:, 4] = c.full[1, 6] = c.full[3, 8] = -1
        c.check()
    # nothing but absent pages
    c = Case([2], [32], [40, 50], 4, 2, 16, seed=13)
    c.bt.fill_(-1)
    assert bool((S.shared_prefix_decode_attn(*c.args()) == 0).all())


def test_lengths_beyond_the_table_and_negative():
    c = Case([3], [32], [64, 64, 40], 8, 2, 16, seed=14)
    a = list(c.args())
    a[4] = torch.tensor([64, 1000, 40], dtype=torch.int32, device=DEV)      # (the table holds 64)
    c.check(got=S.shared_prefix_decode_attn(*a))
    a[4] = torch.tensor([64, 64, -7], dtype=torch.int32, device=DEV)
    c.lens = [64, 64, 0]
    c.check(got=S.shared_prefix_decode_attn(*a))


@pytest.mark.parametrize("scale", [0.0, -0.05, 3.0])
def test_scales(scale):
    c = Case([5], [300], rng_lens(15, [5], [300], 1, 50), 8, 2, 16, seed=15)
    c.check(scale=scale)
    c.check(BF16, scale=scale)


def test_far_logits():
    # one token far above the rest, in the shared part for some rows, in the own part for others
    c = Case([4], [256], [300, 310, 290, 270], 8, 2, 16, seed=16)
    for b, t in ((0, 40), (1, 305), (2, 255), (3, 0)):
        for h in range(2):
            c.k[int(c.full[b, t // 16]), h, t % 16] = (c.q[b, 4 * h] * 8).to(torch.bfloat16)
    c.check()
    c.check(BF16)


def test_many_groups_and_sequences():
    log("case shared many")
    per = [2, 1, 3] * 300
    pre = [16, 50, 33] * 300
    Case(per, pre, rng_lens(17, per, pre, 0, 20), 2, 1, 16, seed=17, nan=False).check()
    Case([], [], [5] * 8192, 1, 1, 16, seed=18, nan=False).check()


def test_the_most_groups():
    n = S.SPARROW_MAX_GROUPS
    per, pre = [2] * n, [16] * n
    c = Case(per, pre, [20] * (2 * n), 1, 1, 16, seed=19, nan=False)
    c.check()
    a = list(c.args())
    a[5] = torch.zeros(n + 2, dtype=torch.int32, device=DEV)
    a[6] = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
    with pytest.raises(S.SparrowError):
        S.shared_prefix_decode_attn(*a)


def test_repeated_calls_are_equal():
    per, pre = [16, 16], [2000, 1500]
    c = Case(per, pre, rng_lens(20, per, pre, 1, 400), 8, 2, 16, seed=20, nan=False)
    a = c.args()
    x = S.shared_prefix_decode_attn(*a)
    for _ in range(3):
        assert torch.equal(S.shared_prefix_decode_attn(*a), x)


def test_no_sequences():
    q = torch.zeros((0, 4, D), dtype=torch.bfloat16, device=DEV)
    k = torch.zeros((1, 2, 16, D), dtype=torch.bfloat16, device=DEV)
    i = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = S.shared_prefix_decode_attn(q, k, k, torch.zeros((0, 3), dtype=torch.int32, device=DEV), i[:0],
                                      i, i[:0])
    assert out.shape == (0, 4, D)


def test_wrapper_refusals():
    c = Case([2], [32], [40, 50], 4, 2, 16, seed=21)
    ok = list(c.args())

    def bad(i, t, **kw):
        a = list(ok)
        a[i] = t
        with pytest.raises((ValueError, RuntimeError)):
            S.shared_prefix_decode_attn(*a, **kw)
    bad(0, ok[0].float())
    bad(0, ok[0][:, :3].contiguous())
    bad(1, ok[1].float())
    bad(1, ok[1].transpose(1, 2))
    bad(2, ok[2][:3])
    bad(3, ok[3].long())
    bad(3, ok[3][:, ::2])
    bad(4, ok[4].long())
    bad(4, ok[4].cpu())
    bad(5, ok[5][:1])
    bad(5, ok[5].long())
    bad(6, ok[6].long())
    bad(6, ok[6][:, None])
    bad(6, ok[6].cpu())
    bad(0, ok[0], out=torch.empty((2, 4, D), dtype=torch.bfloat16, device=DEV))
    bad(0, ok[0], out_dtype=7)
    bad(0, ok[0], scale=math.nan)
    bad(0, ok[0], workspace=torch.empty(64, dtype=torch.uint8, device=DEV))


def test_side_stream_and_graph_replays():
    per, pre = [8, 5], [700, 90]
    c = Case(per, pre, rng_lens(22, per, pre, 1, 100), 8, 2, 16, seed=22, nan=False)
    a = c.args()
    want = S.shared_prefix_decode_attn(*a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    sh = S.make_shape(13, 8, 2, 16, a[3].shape[1], a[1].shape[0])
    ws = torch.empty(S.sparrow_shared_prefix_workspace_size(sh, 2), dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(want)
    with torch.cuda.stream(side):
        assert torch.equal(S.shared_prefix_decode_attn(*a), want)
        with torch.cuda.graph(graph, stream=side):
            S.shared_prefix_decode_attn(*a, out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        if rep == 2:                                    # the sequences go on, the same graph
            a[4].sub_(1)
            want = S.shared_prefix_decode_attn(*a)
        out.fill_(math.nan)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), rep


def test_two_calls_at_once():
    cs = [Case([8], [4000], rng_lens(23 + i, [8], [4000], 1, 100), 8, 2, 16, seed=23 + i, nan=False)
          for i in range(2)]
    args = [c.args() for c in cs]
    want = [S.shared_prefix_decode_attn(*a) for a in args]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(S.shared_prefix_decode_attn(*args[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_offsets_past_32_bits():
    # the pages lie behind 2^32 bytes and 2^31 elements of a cache, one sequence on the last of them
    hkv, ps = 2, 128
    P = (5 << 30) // (hkv * ps * D * 2)
    k = torch.empty((P, hkv, ps, D), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    c = Case([3], [300], [310, 400, 384], 8, hkv, ps, seed=30, nan=False)
    n = c.k.shape[0]
    k[P - n:] = c.k.to(DEV)
    v[P - n:] = c.v.to(DEV)
    a = list(c.args())
    a[1], a[2], a[3] = k, v, a[3] + (P - n)
    c.check(got=S.shared_prefix_decode_attn(*a))
