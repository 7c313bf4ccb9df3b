"""Attention over an e4m3 cache where a wave takes more than one batch of 64 pages of a list: over 65536
(page, KV head) pairs in a call.  Every (sequence, KV head) against the formula in 64 bits.

Tolerance, in units of sum_t w_t |v_t|: a logit is a sum of 128 exact products in fp32, off by at most
2^-17 of scale sum |q k|, and so is a weight's logarithm, in the numerator and in the sum: 2^-16 of the
largest scale sum |q k_t|.  A wave's state goes through at most some 90 tiles here, each with a rescaling
and three additions, 2^-23 each, and a unit's through at most 8 waves: 2^-14.  Then one rounding of the
output, 2^-24."""
import math

import numpy as np
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
D = 128
HKV = 8


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


class Long:
    """Ragged sequences of about 64 n pages, n not whole, in a cache of random rows; NaN codes and the
    largest exponents wherever no token is."""

    def __init__(self, seed, hq, ps, pages):
        g = self.g = np.random.default_rng(seed)
        self.hq, self.ps, self.pages = hq, ps, np.array(pages)
        # whole last pages, one token in it, and others
        self.lens = self.pages * ps - np.where(g.random(len(pages)) < 0.3, 0,
                                               g.choice([ps - 1, 1, ps // 2], len(pages)))
        P = int(self.pages.sum()) + 3
        perm = g.permutation(P)
        bt = np.full((len(pages), int(self.pages.max()) + 1), -1, np.int32)
        at = 0
        for b, n in enumerate(pages):
            bt[b, :n] = perm[at:at + n]
            at += n
        self.bt = torch.from_numpy(bt).to(DEV)
        self.seq_lens = torch.from_numpy(self.lens.astype(np.int32)).to(DEV)
        held = np.zeros(P, np.int64)                        # tokens in each physical page
        for b, L in enumerate(self.lens):
            held[bt[b, :pages[b]]] = np.minimum(ps, L - ps * np.arange(pages[b]))
        dead = torch.arange(ps, device=DEV)[None] >= torch.from_numpy(held).to(DEV)[:, None]
        dead = dead[:, None].expand(P, HKV, ps)
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.k8, self.v8, self.exps = S.new_cache_e4m3(P, HKV, ps, DEV)
        for j, c in enumerate((self.k8, self.v8)):
            c.copy_(torch.randn(c.shape, generator=gen, device=DEV, dtype=torch.bfloat16))
            c.view(torch.uint8)[dead] = 0x7f
            e = torch.randint(123, 128, (P, HKV, ps), generator=gen, device=DEV).to(torch.uint8)
            e[dead] = 255
            self.exps[:, :, :, j] = e.view(P, HKV, ps // 4, 4)
        self.q = torch.randn((len(pages), hq, D), generator=gen, device=DEV).to(torch.bfloat16)

    def rows(self, codes, j, phys, h, seen):
        x = codes.view(torch.uint8)[phys, h].view(torch.float8_e4m3fn).float().double()
        e = self.exps[phys, h][:, :, j].reshape(len(phys), self.ps, 1).double()
        return (x * torch.exp2(e - 127)).flatten(0, 1)[seen]

    def check(self, got, lists, what):
        """``lists``: a unit's logical pages, by sequence and KV head."""
        G, scale, worst = self.hq // HKV, 1 / math.sqrt(D), 0.0
        for b, L in enumerate(self.lens):
            for h in range(HKV):
                pages = torch.from_numpy(np.asarray(lists(b, h))).to(DEV)
                seen = (pages[:, None] * self.ps + torch.arange(self.ps, device=DEV)).flatten() < int(L)
                phys = self.bt[b].long()[pages]
                k, v = self.rows(self.k8, 0, phys, h, seen), self.rows(self.v8, 1, phys, h, seen)
                q = self.q[b, h * G:(h + 1) * G].double()
                w = torch.softmax(scale * torch.matmul(q, k.t().contiguous()), -1)
                far = scale * torch.matmul(q.abs(), k.abs().t().contiguous()).amax(-1, keepdim=True)
                want, size = torch.matmul(w, v), torch.matmul(w, v.abs())
                err = (got[b, h * G:(h + 1) * G].double() - want).abs()
                tol = (2.0 ** -16 * far + 2.0 ** -14) * size + 2.0 ** -24 * want.abs()
                worst = max(worst, float((err / tol).max()))
                assert bool((err <= tol).all()), (what, b, h, int(L), float((err / tol).max()))
        log(f"{what}: at most {worst:.3f} of the tolerance")


# lists of 0, 1 and 63 pages past a whole number of batches, and others
PAGES = [256, 257, 319, 320, 321, 383, 64, 65, 127, 449] * 3 + [300, 281, 266, 299, 310, 290, 277, 333, 350, 290]


@pytest.mark.parametrize("hq,ps", [(16, 16), (80, 16), (128, 32)])
def test_dense(hq, ps):
    log(f"case e4m3 long dense heads={hq} ps={ps}")
    c = Long(hq + ps, hq, ps, PAGES)
    assert c.pages.sum() * HKV > 65536
    out = S.dense_decode_attn_e4m3(c.q, c.k8, c.v8, c.exps, c.bt, c.seq_lens)
    c.check(out, lambda b, h: np.arange(c.pages[b]), "dense")


@pytest.mark.parametrize("hq,ps,ordered", [(32, 16, True), (16, 32, False)])
def test_sparse(hq, ps, ordered):
    log(f"case e4m3 long sparse heads={hq} ps={ps}")
    c = Long(hq + ps, hq, ps, [n + 7 for n in PAGES])
    counts = np.array(PAGES)
    assert counts.sum() * HKV > 65536
    idx = np.full((len(PAGES), HKV, 460), -1, np.int32)
    for b, n in enumerate(counts):
        for h in range(HKV):
            pick = c.g.permutation(c.pages[b])[:n]
            idx[b, h, :n] = np.sort(pick) if ordered else pick
    out = S.sparse_decode_attn_e4m3(c.q, c.k8, c.v8, c.exps, c.bt, c.seq_lens,
                                    torch.from_numpy(counts.astype(np.int32)).to(DEV),
                                    torch.from_numpy(idx).to(DEV))
    c.check(out, lambda b, h: idx[b, h, :counts[b]].astype(np.int64), "sparse")
