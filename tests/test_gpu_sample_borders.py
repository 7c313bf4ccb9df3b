"""Token sampling without filters where a draw falls on a border between spans, the next one's first block masked."""
import math

import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


@pytest.mark.parametrize("dtype", [F32, BF])
def test_draw_on_a_border_before_a_masked_block(dtype):
    # Both halves of a row are the same 32 spans, and u = 1/2: the draw is the sum of the first half exactly.
    # The running sum in front of the second half, from other roundings, may come out above it, by a
    # step; the second half's first block is masked and may not be drawn for that.
    E = 1024 if dtype == F32 else 2048      # tokens of a span of 256 vectors, four blocks
    T, V = 400, 64 * E
    log(f"case sample border V={V} {dtype}")
    g = torch.Generator().manual_seed(5)
    half = torch.randn((T, V // 2), generator=g)
    half[:, :E // 4] = -math.inf
    z = torch.cat([half, half], 1).to(dtype)
    u = torch.full((T,), 0.5)
    tok, lp = (t.cpu() for t in S.sample(z.to(DEV), u.to(DEV)))
    rows = torch.arange(T)
    assert bool(((tok >= 0) & (tok < V)).all()), tok.min()
    drawn = z.double()[rows, tok.long()]
    assert bool((drawn > -math.inf).all()), torch.nonzero(drawn == -math.inf).flatten().tolist()[:8]
    w = z.double().exp()
    c = w.cumsum(1)
    total = c[:, -1]
    # the border itself, to the 1e-13 that sums are held to and 1e-11 for this running sum
    assert bool((c[rows, tok.long()] >= total * (0.5 - 1e-10)).all())
    assert bool((c[rows, tok.long()] - w[rows, tok.long()] <= total * (0.5 + 1e-10)).all())
    want = drawn - total.log()
    assert bool(((lp.double() - want).abs() <= 2.0 ** -24 * want.abs() + 1e-11).all())


def test_a_kept_token_of_no_weight_is_not_drawn():
    # The same border among tokens that are sorted: two equal halves of 64, the first token of each, and some others,
    # so far below the rest that their weights are 0 in 64 bits.  They stay in top-k, and may not be drawn.
    T, V = 600, 200
    log("case sample border of kept tokens")
    g = torch.Generator().manual_seed(6)
    half = torch.randn((T, 64), generator=g)
    half[torch.rand((T, 64), generator=g) < 0.2] = -3e4
    half[:, 0] = -3e4
    z = torch.full((T, V), -math.inf)
    z[:, :128] = torch.cat([half, half], 1)
    u = torch.full((T,), 0.5)
    for kw in (dict(top_k=torch.full((T,), 128, dtype=torch.int32)), dict(top_p=torch.full((T,), 0.999999))):
        tok, lp = (t.cpu() for t in S.sample(z.to(DEV), u.to(DEV), **{k: v.to(DEV) for k, v in kw.items()}))
        drawn = z.double()[torch.arange(T), tok.long()]
        assert bool((drawn > -1e4).all()), (list(kw), torch.nonzero(drawn <= -1e4).flatten().tolist()[:8])
        assert bool(lp.isfinite().all())
