"""Numbers that are not finite in decode attention over shared prefixes: they reach the rows that attend to them and no
others, against the definition and the dense operator on full tables."""
import math

import numpy as np
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log
from test_gpu_attention_shared import BF16, D, DEV, F32, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


def dense(c, dtype=F32, **kw):
    """The dense operator on tables that name every token's own page."""
    a = c.args()
    full = torch.from_numpy(c.full.astype(np.int32)).to(DEV)
    return S.dense_decode_attn(*a[:3], full, a[4], out_dtype=dtype, **kw)


@pytest.mark.parametrize("where", ["shared", "own", "query"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logits_that_are_no_number(where, dtype):
    # rows that attend to them hold no number, and no other row does (the dense operator's do for such a key, but
    # it gives a row of zeros for such a query)
    for ps, hq, hkv in ((16, 8, 2), (64, 5, 1)):
        log(f"case shared NaN logits {where} ps={ps} out={dtype}")
        lens = [210, 30, 250, 0, 193, 70]
        c = Case([5, 1], [192, 20], lens, hq, hkv, ps, seed=3)
        hit = torch.zeros((6, hq), dtype=torch.bool)
        if where == "shared":
            c.k[int(c.full[0, 50 // ps]), 0, 50 % ps, 11] = math.nan
            hit[[0, 2, 4], :hq // hkv] = True
        elif where == "own":
            c.k[int(c.full[2, 249 // ps]), 0, 249 % ps, 3] = math.nan
            hit[2, :hq // hkv] = True
        else:
            c.q[4, 1, 100] = math.nan
            hit[4, 1] = True
        got, other = S.shared_prefix_decode_attn(*c.args(), out_dtype=dtype), dense(c, dtype)
        assert torch.equal(got.isnan().cpu(), hit[..., None].expand(-1, -1, D))
        assert where == "query" or torch.equal(got.isnan(), other.isnan())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("hq,hkv,ps", [(8, 2, 16), (2, 1, 32), (32, 2, 64)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sequences_that_end_before_a_v_that_is_not_finite(bad, hq, hkv, ps, dtype):
    # the shared tokens from `at` on; sequences that end before are as without it, the others hold it
    for at in (0, 1, 5, 31, 32, 100, 170):
        log(f"case shared V={bad} at={at} heads={hq},{hkv} ps={ps} out={dtype}")
        lens = [200, at, 195, max(0, at - 1), 192 + at % 7, at // 2, at + 1, 0, at, 300]
        c = Case([9, 1], [192, 10], lens, hq, hkv, ps, seed=at)
        want, size, most = c.reference(1 / math.sqrt(D))
        c.v[int(c.full[0, at // ps]), :, at % ps, ::3] = bad
        if at % 2:
            c.v[int(c.full[0, 180 // ps]), 0, 180 % ps, 7] = -bad
        got = S.shared_prefix_decode_attn(*c.args(), out_dtype=dtype)
        other = dense(c, dtype)
        before = [b for b, n in enumerate(lens) if n <= at or b == 9]
        tol = (2 * 2 ** -17.5 * most + 2 ** -14) * size + 1e-30
        if dtype == BF16:
            tol = tol + 2 ** -7 * size + 2 ** -8 * want.abs()
        assert bool(((got.cpu().double() - want).abs() <= tol)[before].all())
        # (a weight of 0 times an infinite V is no number on either side, so weights matter only as far as that)
        behind = [b for b in range(10) if b not in before]
        assert torch.equal(got[behind].isfinite(), other[behind].isfinite())
        assert not bool(got[behind][..., ::3].isfinite().any())
