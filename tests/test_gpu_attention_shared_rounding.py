"""Decode attention over shared prefixes rounds once: a bf16 output is the fp32 one rounded, and holds the softmax
numerators' 24 bits as far as its own type does."""
import math

import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log
from test_gpu_attention_shared import BF16, D, F32, GROUPS, Case, rng_lens

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


@pytest.mark.parametrize("per,pre,lo,hi", GROUPS)
@pytest.mark.parametrize("hq,hkv,ps", [(8, 2, 32), (3, 3, 16)])
def test_a_bf16_output_is_the_fp32_one_rounded(per, pre, lo, hi, hq, hkv, ps):
    log(f"case shared rounded per={per} pre={pre} heads={hq},{hkv} ps={ps}")
    c = Case(per, pre, rng_lens(sum(per) + ps, per, pre, lo, hi), hq, hkv, ps, seed=sum(pre))
    wide = S.shared_prefix_decode_attn(*c.args(), out_dtype=F32)
    assert torch.equal(S.shared_prefix_decode_attn(*c.args(), out_dtype=BF16), wide.to(torch.bfloat16))


@pytest.mark.parametrize("per,pre,lens", [([2], [16], [20, 17]), ([3], [40], [45, 41, 60]), ([8], [300], [310] * 8)])
def test_a_bf16_output_has_one_rounding(per, pre, lens):
    # the fp32 output's bound (numerator and denominator 2^-17.5 Z each, 2^-14 for exponential and sums) and half
    # a step of the output's type: no room for numerators of 8 bits
    log(f"case shared one rounding per={per}")
    c = Case(per, pre, lens, 8, 2, 16, seed=sum(lens))
    want, size, most = c.reference(1 / math.sqrt(D))
    got = S.shared_prefix_decode_attn(*c.args(), out_dtype=BF16).cpu().double()
    tol = (2 * 2 ** -17.5 * most + 2 ** -14) * size
    assert bool(((got - want).abs() <= tol + 2 ** -8 * (want.abs() + tol)).all())
