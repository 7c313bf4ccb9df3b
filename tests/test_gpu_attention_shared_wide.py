"""Decode attention over shared prefixes on a table so wide that a position of its plan is several tiles."""
import math

import numpy as np
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
D = 128


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield
    torch.cuda.empty_cache()


def test_several_tiles_a_position():
    # 8192 sequences of 7 heads on a table for the longest: 2^31 positions of one tile would not do, so one is
    # two.  Own tokens end on odd and even tiles, in the first half of a tile and in the second.
    B, hkv, ps, M = 8192, 7, 128, S.SPARROW_MAX_PAGES_PER_SEQ
    tiles = M * ps // 32
    assert (tiles + 3) * hkv * B > 2 ** 31
    log("case shared wide table")
    g = torch.Generator().manual_seed(41)
    per = [5, 3, 1, 70]
    cu, pre = np.cumsum([0] + per), [700, 130, 300, 257]
    lens = torch.zeros(B, dtype=torch.int64)
    many = torch.randint(0, B, (500,), generator=g)
    lens[many] = torch.randint(1, 400, (500,), generator=g)
    lens[:80] = torch.randint(1, 400, (80,), generator=g)
    for i, n in enumerate(per):
        lens[cu[i]:cu[i + 1]] += pre[i]
    lens[3], lens[cu[1]] = 100, 0                 # ended, and never begun
    P = 400
    k, v = (torch.randn((P, hkv, ps, D), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    q = torch.randn((B, hkv, D), generator=g).to(torch.bfloat16).to(DEV)
    narrow = torch.randint(0, P, (B, 12), generator=g, dtype=torch.int32)
    for i, n in enumerate(per):
        narrow[cu[i]:cu[i + 1], :pre[i] // ps] = narrow[cu[i], :pre[i] // ps].clone()
    narrow = narrow.to(DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    lens_d, cu_d, pre_d = lens.to(**i32), torch.tensor(cu, **i32), torch.tensor(pre, **i32)
    small = S.shared_prefix_decode_attn(q, k, v, narrow, lens_d, cu_d, pre_d)
    table = torch.full((B, M), -1, **i32)
    table[:, :12] = narrow
    large = S.shared_prefix_decode_attn(q, k, v, table, lens_d, cu_d, pre_d)
    # against the formula for every sequence with a token, and between the two splits of the work
    rows = torch.nonzero(lens > 0).flatten()
    kd, vd, qd, bt = k.cpu().double(), v.cpu().double(), q.cpu().double(), narrow.cpu().long()
    for b in rows.tolist():
        at = torch.arange(int(lens[b]))
        page = bt[b][at // ps]
        kk, vv = kd[page, :, at % ps].transpose(0, 1), vd[page, :, at % ps].transpose(0, 1)
        w = torch.softmax((kk @ qd[b][..., None]).squeeze(-1) / math.sqrt(D), -1)
        want, size = (w[:, None] @ vv)[:, 0], (w[:, None] @ vv.abs())[:, 0]
        most = ((kk.abs() @ qd[b].abs()[..., None]).amax() / math.sqrt(D))
        tol = (2 * 2 ** -17.5 * most + 2 ** -14) * size
        for got in (large, small):
            assert bool(((got[b].cpu().double() - want).abs() <= tol).all()), b
    assert bool((large[lens.to(DEV) == 0] == 0).all())
