"""The head norms and their gradient on texts that fill the GPU many times over, and every output at small
and large scales, against the formulas in 64 bits (on the GPU, some tokens at a time).

Tolerances of y and dx as for the short texts: one rounding to bf16 (2^-8 of the value) and 2^-18 of
|n_i| + |n_{i+64}|, 2^-17 of the sum of the gradient's terms.  A weight's gradient: its terms are off by at
most 2^-19 of theirs (r 2^-20, sine and cosine 2^-23, products); a lane adds up n of them one after another, and
then at most 40 sums of lanes, waves and workgroups, 2^-24 of the sum of magnitudes each."""
import numpy as np
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
D = 128
EPS = 1e-6


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


def turn(x, f, pos, sign=1):
    """The rotation of [T][h][128] in 64 bits, and the size of the terms it adds."""
    a = sign * pos.double()[:, None, None] * f
    lo, hi = x[..., :64], x[..., 64:]
    size = lo.abs() + hi.abs()
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1), \
        torch.cat([size, size], -1)


def formula(x, w, f, pos):
    x = x.double()
    return turn(x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w.double(), f, pos)


def formula_grad(dy, x, w, f, pos):
    x, w = x.double(), w.double()
    r = 1 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
    g, size = turn(dy.double(), f, pos, -1)
    xn = x * r
    dx = r * (g * w - xn * (g * w * xn).mean(-1, keepdim=True))
    dxs = r * (size * w.abs() + xn.abs() * (size * w.abs() * xn.abs()).mean(-1, keepdim=True))
    return dx, dxs, (g * xn).sum((0, 1)), (size * xn.abs()).sum((0, 1))


def check(got, want, size, part, what):
    err = (got.double() - want).abs()
    over = err - (2.0 ** -8 * want.abs() + part * size)
    assert bool((over <= 0).all()), (what, float(over.max()), float(err.max()))


def make(T, hq, hk, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    q, k = (torch.randn((T, h, D), generator=g, device=DEV, dtype=torch.bfloat16) for h in (hq, hk))
    w = [(1 + 0.3 * torch.randn(D, generator=g, device=DEV)).to(torch.bfloat16) for _ in range(2)]
    f = torch.from_numpy(1e6 ** (-np.arange(0, D, 2) / D)).to(DEV)
    pos = torch.randint(0, 40000, (T,), generator=g, device=DEV, dtype=torch.int32)
    pos[torch.rand(T, generator=g, device=DEV) < 0.01] = -1
    return q, k, w, f, pos


# Waves of each side and the additions of a lane follow from 512 workgroups of 4 waves, shared out by the
# sides' passes of 8 heads: 70000 tokens in 1924 (query) and 124 (key) waves are 37 tokens of 16 passes and
# 565 of one; 80000 in 1536 and 512 are 53 of 3 and 157 of one.  (2.3 GB and 655 MB of rows, so that both
# are stored past the caches.)
@pytest.mark.parametrize("T,hq,hk,adds", [(70000, 128, 2, (592, 565)), (80000, 24, 8, (159, 157))])
def test_streamed_gradient(T, hq, hk, adds):
    log(f"case rope long gradient T={T} heads={hq},{hk}")
    q, k, w, f, pos = make(T, hq, hk, T + hq)
    # a gradient along the output: every term of dw is then positive, and none may be missing
    y = [torch.zeros_like(t) for t in (q, k)]
    S.qk_norm_rope(q, k, w[0], w[1], f, pos, EPS, q_out=y[0], k_out=y[1])
    for t in (q, k, *y):
        t[pos < 0] = float("nan")
    out = S.qk_norm_rope_bwd(y[0], y[1], q, k, w[0], w[1], f, pos, EPS)
    for i, x in enumerate((q, k)):
        dw, size = torch.zeros(D, dtype=torch.float64, device=DEV), torch.zeros(D, dtype=torch.float64, device=DEV)
        for at in torch.arange(T, device=DEV).split(max(1, 400000 // x.shape[1])):
            assert bool((out[i][at][pos[at] < 0] == 0).all())
            at = at[pos[at] >= 0]
            dx, dxs, part, ps = formula_grad(y[i][at], x[at], w[i], f, pos[at])
            check(out[i][at], dx, dxs, 2.0 ** -17, "dx")
            dw, size = dw + part, size + ps
        err = ((out[2 + i].double() - dw).abs() / size).max()
        log(f"weight {i}: {float(err):.2e} of the sum of magnitudes")
        assert float(err) <= 2.0 ** -19 + (adds[i] + 40) * 2.0 ** -24


def test_forward_beyond_the_grid():
    # more than 2^20 workgroups of 4 waves, a wave per token and side: from token 2^21 on a workgroup's second turn
    T, cap = 2200003, 1 << 21
    q, k, w, f, pos = make(T, 1, 1, 7)
    pos[cap - 3:cap - 1] = -1
    pos[cap + 1:cap + 3] = -1
    pos[cap] = pos[cap - 1] = pos[T - 1] = 39999
    outs = [torch.full_like(t, 7.0) for t in (q, k)]
    S.qk_norm_rope(q, k, w[0], w[1], f, pos, EPS, q_out=outs[0], k_out=outs[1])
    for got, x, wt in zip(outs, (q, k), w):
        assert bool((got[pos < 0] == 7).all())
        for at in torch.arange(T, device=DEV).split(400000):
            at = at[pos[at] >= 0]
            check(got[at], *formula(x[at], wt, f, pos[at]), 2.0 ** -18, "beyond the grid")


@pytest.mark.parametrize("scale", [1e-20, 1e-3, 1e12])
def test_every_output_at_small_and_large_scales(scale):
    q, k, w, f, pos = make(6, 4, 2, 9)
    pos.abs_()
    q, k = q * scale, k * scale
    q[2] = 0
    k[3] = 0
    g = torch.Generator(device=DEV).manual_seed(10)
    dy = [torch.randn(t.shape, generator=g, device=DEV).to(torch.bfloat16) for t in (q, k)]
    y = S.qk_norm_rope(q, k, w[0], w[1], f, pos, EPS)
    out = S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos, EPS)
    for i, x in enumerate((q, k)):
        check(y[i], *formula(x, w[i], f, pos), 2.0 ** -18, "y")
        dx, dxs, dw, size = formula_grad(dy[i], x, w[i], f, pos)
        check(out[i], dx, dxs, 2.0 ** -17, "dx")
        err = (out[2 + i].double() - dw).abs()
        assert bool((err <= (2.0 ** -19 + 50 * 2.0 ** -24) * size).all()), float((err / size).max())
