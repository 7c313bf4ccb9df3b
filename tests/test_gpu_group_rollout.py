"""Decode steps of a grouped rollout: several samples of every prompt, one token each a step, through a small
model of two layers: norm, projection, per-head norm and rotation, append, attention over the groups' shared
prefixes, projection, the norms around the gated block, the head's logits, the next tokens.

Every operator's result is checked against the formula in 64 bits on what it read, with the tolerances
of its own tests, and the run as a whole: eager, in other workspaces and on another stream, and as one captured
step replayed."""
import math

import numpy as np
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log
from test_gpu_qk_norm_rope import check as check_rope, formula as rope
from test_gpu_residual_norm import check_forward as check_norm
from test_gpu_sample import check as check_tokens

pytestmark = pytest.mark.gpu

DEV = "cuda"
D = 128
BF = torch.bfloat16
EPS = 1e-6
SCALE = 1 / math.sqrt(D)


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


class Rollout:
    """Groups of `per` samples of prompts of `pre` tokens, `steps` tokens of room; hq, hkv heads."""

    def __init__(self, per, pre, steps, hq=6, hkv=2, C=520, V=1003, ps=16, layers=2, seed=0,
                 stream=BF):
        g = torch.Generator().manual_seed(seed)

        def randn(*shape, by=1.0):
            return (torch.randn(shape, generator=g) * by).to(BF).to(DEV)
        B = sum(per)
        self.B, self.hq, self.hkv, self.C, self.V, self.ps, self.per, self.pre = \
            B, hq, hkv, C, V, ps, per, pre
        shared = [p // ps for p in pre]
        own = [-(-(p + steps) // ps) - s for p, s in zip(pre, shared)]
        M = max(s + o for s, o in zip(shared, own))
        P = sum(s + n * o for n, s, o in zip(per, shared, own))
        page = torch.randperm(P, generator=g).tolist()
        bt = np.full((B, M), -1, np.int32)
        b = 0
        for n, s, o in zip(per, shared, own):
            first = [page.pop() for _ in range(s)]
            for _ in range(n):
                bt[b, :s] = first
                bt[b, s:s + o] = [page.pop() for _ in range(o)]
                b += 1
        i32 = dict(dtype=torch.int32, device=DEV)
        self.bt = torch.from_numpy(bt).to(DEV)
        self.cu = torch.tensor([0] + np.cumsum(per).tolist(), **i32)
        self.prefix = torch.tensor(pre, **i32)
        self.start = torch.tensor(np.repeat(pre, per), **i32)   # (the prompts' tokens are in the caches)
        self.prompts = [[randn(P, hkv, ps, D) for _ in range(2)] for _ in range(layers)]
        for n, p, first in zip(per, pre, np.cumsum([0] + per)):  # a part of a page: every sample its own
            rest = p % ps
            for k, v in self.prompts:
                for b in range(first, first + n):
                    if rest:
                        at, to = bt[first, p // ps], bt[b, p // ps]
                        k[to, :, :rest], v[to, :, :rest] = k[at, :, :rest].clone(), \
                            v[at, :, :rest].clone()
        H = hq + 2 * hkv
        self.embed = randn(V, C)
        self.w_in = [randn(C, H * D, by=C ** -0.5) for _ in range(layers)]
        self.w_out = [randn(hq * D, 2 * C, by=(hq * D) ** -0.5) for _ in range(layers)]
        self.head = randn(C, V, by=3 * C ** -0.5)
        self.norms = [(1 + randn(C, by=0.2)).to(BF) for _ in range(layers + 1)]
        self.post = [(1 + randn(C, by=0.2)).to(BF) for _ in range(layers)]
        self.head_norms = [(1 + randn(D, by=0.2)).to(BF) for _ in range(2)]
        self.freq = torch.from_numpy(1e6 ** (-np.arange(0, D, 2) / D)).to(DEV)
        self.stream = stream
        self.u = torch.rand((steps, B), generator=g).to(DEV)
        self.temp = (0.6 + 0.6 * torch.rand(B, generator=g)).to(DEV)
        self.k = torch.randint(0, 50, (B,), generator=g, dtype=torch.int32).to(DEV)
        self.p = (0.7 + 0.35 * torch.rand(B, generator=g)).to(DEV)
        self.reset()

    def reset(self):
        self.caches = [[t.clone() for t in kv] for kv in self.prompts]
        self.meta = [S.new_meta(kv[0].shape[0], self.hkv, DEV) for kv in self.prompts]
        self.lens = self.start.clone()
        self.tokens = (torch.arange(self.B, device=DEV, dtype=torch.int32) * 7) % self.V

    def step(self, u, seen=None):
        """One token of every sample; `seen` gathers what the operators read and wrote."""
        self.lens += 1
        pos = self.lens - 1
        h = self.embed[self.tokens.long()].to(self.stream)
        h, y = S.residual_norm(h, None, self.norms[0], eps=EPS)
        ops = [("norm", dict(h=h, x=None, weight=self.norms[0], post_weight=None, gate=None, scale=1.0,
                             eps=EPS), (h, y))]
        for i, (kc, vc) in enumerate(self.caches):
            qkv = y @ self.w_in[i]
            n = self.hq * D
            q = qkv[:, :n].unflatten(1, (self.hq, D))
            k = qkv[:, n:n + self.hkv * D].unflatten(1, (self.hkv, D))
            v = qkv[:, n + self.hkv * D:].unflatten(1, (self.hkv, D)).contiguous()
            qr, kr = S.qk_norm_rope(q, k, *self.head_norms, self.freq, pos, EPS)
            ops.append(("rope", (q, k, self.head_norms, self.freq, pos, EPS), (qr, kr)))
            S.append_kv(kr, v, kc, vc, self.bt, self.lens, self.meta[i])
            out = S.shared_prefix_decode_attn(qr, kc, vc, self.bt, self.lens, self.cu, self.prefix,
                                              out_dtype=S.SPARROW_OUT_BF16)
            ops.append(("attention", (qr, i, kr, v), out))
            x, gate = (out.flatten(1) @ self.w_out[i]).split(self.C, 1)
            d = dict(h=h, x=x, weight=self.norms[i + 1], post_weight=self.post[i], gate=gate, scale=0.7,
                     eps=EPS)
            h, y = S.residual_norm(**d)
            ops.append(("norm", d, (h, y)))
        z = y @ self.head
        self.tokens, lp = S.sample(z, u, self.temp, self.k, self.p)
        ops.append(("sample", (z, u, self.temp, self.k, self.p), (self.tokens, lp)))
        if seen is not None:
            seen += ops
        return self.tokens, lp, z

    def attention(self, q, layer):
        """(out, sum of |w v|, largest |q||k|) in 64 bits from the caches as they are."""
        k, v = (t.cpu().double() for t in self.caches[layer])
        bt, G = self.bt.cpu().long(), self.hq // self.hkv
        q = q.cpu().double()
        out, size = torch.zeros_like(q), torch.zeros_like(q)
        most = torch.zeros((*q.shape[:2], 1), dtype=torch.float64)
        for b, n in enumerate(self.lens.tolist()):
            at = torch.arange(n)
            page = bt[b][at // self.ps]
            for j in range(self.hkv):
                rows = slice(j * G, (j + 1) * G)
                kk, vv = k[page, j, at % self.ps], v[page, j, at % self.ps]
                w = torch.softmax(SCALE * q[b, rows] @ kk.T, -1)
                out[b, rows], size[b, rows] = w @ vv, w @ vv.abs()
                most[b, rows] = SCALE * (q[b, rows].abs() @ kk.abs().T).amax(-1, keepdim=True)
        return out, size, most

    def check(self, ops):
        pages = (self.lens - 1).long() // self.ps
        page = self.bt[torch.arange(self.B, device=DEV), pages].long()
        slot = (self.lens - 1).long() % self.ps
        for name, args, got in ops:
            if name == "norm":
                check_norm(args, got)
            elif name == "rope":
                q, k, w, f, pos, eps = args
                check_rope(got[0], *rope(q, w[0], f, pos, eps), 2.0 ** -18, "q")
                check_rope(got[1], *rope(k, w[1], f, pos, eps), 2.0 ** -18, "k")
            elif name == "sample":
                z, u, t, k, p = args
                check_tokens(z, u, t, k, p, got=got)
            else:
                q, layer, kr, v = args
                kc, vc = self.caches[layer]
                assert torch.equal(kc[page, :, slot], kr) and torch.equal(vc[page, :, slot], v)
                want, size, most = self.attention(q, layer)
                err = (got.cpu().double() - want).abs()
                tol = (2 * 2 ** -17.5 * most + 2 ** -14 + 2 ** -7) * size + 2 ** -8 * want.abs()
                assert bool((err <= tol).all()), float((err - tol).max())


RUNS = [dict(per=[5, 3], pre=[70, 33]), dict(per=[1], pre=[1], hq=2, hkv=1, C=128, V=7),
        dict(per=[17, 1, 4], pre=[200, 15, 640], hq=8, hkv=2, C=1032, ps=64, stream=torch.float32),
        dict(per=[40], pre=[1030], hq=4, hkv=4, C=512, V=50021, ps=32)]


@pytest.mark.parametrize("run", RUNS)
def test_steps_against_the_formulas(run):
    log(f"case rollout {run}")
    r = Rollout(steps=4, **run)
    for u in r.u:
        seen = []
        r.step(u, seen)
        r.check(seen)


@pytest.mark.parametrize("run", RUNS)
def test_a_captured_step_replayed(run):
    log(f"case rollout graph {run}")
    r = Rollout(steps=20, seed=1, **run)
    want = [tuple(t.clone() for t in r.step(u)) for u in r.u]
    caches = [[t.clone() for t in kv] for kv in r.caches]

    # the same steps once more on another stream, and captured there
    r.reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [tuple(t.clone() for t in r.step(u)) for u in r.u]
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))

    r.reset()
    u, first = r.u[0].clone(), r.tokens
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        r.tokens = first
        tokens, lp, z = r.step(u)
        first.copy_(tokens)                  # (the next replay's tokens)
    first.copy_((torch.arange(r.B, device=DEV, dtype=torch.int32) * 7) % r.V)
    for i, (t0, lp0, z0) in enumerate(want):
        u.copy_(r.u[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, z0) and torch.equal(tokens, t0) and torch.equal(lp, lp0), i
        torch.randn(1000, device=DEV).sum()  # (eager work of the program's own in between)
    for a, b in zip(r.caches, caches):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_samples_of_one_prompt_agree_with_samples_alone():
    # a group's members and the same sequences in groups of one: the same tokens, whose logits are
    # the same up to the attention's order of sums
    log("case rollout grouped and alone")
    r = Rollout(per=[6, 2], pre=[100, 37], steps=3, seed=2)
    grouped = [r.step(u)[2].clone() for u in r.u[:1]]
    r.reset()
    r.cu = torch.arange(9, dtype=torch.int32, device=DEV)
    r.prefix = r.start.clone()
    alone = [r.step(u)[2] for u in r.u[:1]]
    for a, b in zip(grouped, alone):
        # two layers of bf16 activations: some 20 roundings of 2^-8 on logits of the order of 3
        assert float((a.double() - b.double()).abs().max()) < 20 * 2 ** -8 * 3
