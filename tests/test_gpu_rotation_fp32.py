"""The rotation's sine and cosine as the fp32 gradient of a weight shows them.

A head of ones has r = 1 (eps = 0), and dy = 1 in the upper half alone makes the weight's gradient
(sin a_i, cos a_i).  Absolute error: the angle is reduced in fp64 to at most pi / 4 and rounded once
(2^-25), the sine's and cosine's last additions are rounded once (values below 1: 2^-25), and what is
added there (below 1/2 in size, with its own roundings of 2^-26 each, three at most) 2^-25 more at most:
3 * 2^-25 < 2^-23.4.  r is read off channel 64 with frequency 0, whose cosine is 1; where it is not
1 the products may be off by 2^-24 more."""
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


def test_sine_and_cosine_to_fp32():
    g = np.random.default_rng(0)
    x = torch.ones((1, 1, D), dtype=torch.bfloat16, device=DEV)
    dy = torch.zeros_like(x)
    dy[..., 64:] = 1
    w = torch.ones(D, dtype=torch.bfloat16, device=DEV)
    worst = 0.0
    for rep in range(64):
        f = g.uniform(0, 2 * np.pi, 64)
        f[0] = 0.0
        if rep == 0:      # angles at and beside every eighth of a turn
            f[1:] = np.arange(63) * np.pi / 4 * (1 + g.choice([0, 2.0 ** -26, -2.0 ** -26], 63))
        pos = 1 if rep < 32 else int(g.integers(1, 1 << 20))
        out = S.qk_norm_rope_bwd(dy, dy, x, x, w, w, torch.from_numpy(f).to(DEV),
                                 torch.tensor([pos], dtype=torch.int32, device=DEV), 0.0)
        for dw in (t.cpu().double().numpy() for t in out[2:]):
            r = dw[64]
            assert abs(r - 1) <= 2.0 ** -23
            want = np.concatenate([np.sin(pos * f), np.cos(pos * f)]) * r
            err = np.abs(dw - want).max()
            worst = max(worst, err)
            assert err <= 2.0 ** -23.4 + (0 if r == 1 else 2.0 ** -24), (rep, err)
    log(f"largest error of a sine or cosine {worst:.3e}, 2^{np.log2(worst):.2f}")
