"""Samples of one prompt in a group and the same sequences each alone: over several decode steps on the same tokens,
every attention output agrees within the operator's own bounds, and so do the tokens that its logits give."""
import math

import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log
from test_gpu_group_rollout import Rollout
from test_gpu_sample import reference

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


@pytest.mark.parametrize("run", [dict(per=[6, 2], pre=[100, 37]), dict(per=[17, 1, 4], pre=[200, 15, 640], hq=8,
                                                                       C=1032, ps=64, stream=torch.float32)])
def test_grouped_and_alone(run):
    log(f"case rollout grouped and alone {run}")
    r = Rollout(steps=6, seed=3, **run)
    B = r.B
    alone = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    for u in r.u:
        seen = []
        tokens, lp, z = r.step(u, seen)
        for name, args, got in seen:
            if name != "attention":
                continue
            # on the same queries and caches; either side is off by (2 * 2^-17.5 Z + 2^-14) S at most, and by half
            # a step of bf16, 2^-8 of the value, where it is rounded to that
            q, layer = args[:2]
            kc, vc = r.caches[layer]
            wide = [S.shared_prefix_decode_attn(q, kc, vc, r.bt, r.lens, cu, pre)
                    for cu, pre in ((r.cu, r.prefix), (alone, r.start))]
            want, size, most = r.attention(q, layer)
            tol = (2 * 2 ** -17.5 * most + 2 ** -14) * size
            a, b = (t.cpu().double() for t in wide)
            assert bool(((a - b).abs() <= 2 * tol).all())
            assert bool(((a - want).abs() <= tol).all()) and bool(((b - want).abs() <= tol).all())
            assert torch.equal(got, wide[0].to(torch.bfloat16))
        # the tokens: the definition's for these logits
        cols = [x.cpu().double().tolist() for x in (u, r.temp, r.p)]
        for i, row in enumerate(z.double().cpu().numpy()):
            want, want_lp = reference(row, cols[0][i], cols[1][i], int(r.k[i]), cols[2][i])
            assert int(tokens[i]) == want
            assert math.isclose(float(lp[i]), want_lp, rel_tol=2.0 ** -23, abs_tol=1e-12)


def test_the_same_tokens_grouped_and_alone():
    # each with its own caches, fed the same tokens: where the two largest logits are further apart than the two
    # runs' logits, the next tokens are equal
    log("case rollout grouped and alone, own caches")
    r = Rollout(per=[6, 2], pre=[100, 37], steps=4, seed=4)
    r.k.fill_(1)                              # (greedy)
    grouped = []
    for u in r.u:
        before = r.tokens.clone()
        tokens, _, z = r.step(u)
        grouped.append((before, tokens.clone(), z.clone()))
    r.reset()
    r.cu, r.prefix = torch.arange(9, dtype=torch.int32, device=DEV), r.start.clone()
    for u, (before, tokens, z) in zip(r.u, grouped):
        r.tokens = before
        got, _, z2 = r.step(u)
        gap = z.double().topk(2, dim=1)[0]
        gap = gap[:, 0] - gap[:, 1]
        moved = (z.double() - z2.double()).abs().amax(1)
        same = gap > 2 * moved
        assert torch.equal(got[same], tokens[same])
        assert 2 * int(same.sum()) > r.B      # (or little is compared)
