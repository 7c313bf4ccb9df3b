"""Per-head norm with rotation and its gradient against the formulas in 64 bits (on the CPU).

Tolerances.  One rounding to bf16 is off by at most 2^-8 of the value.  In fp32, the turn (half a
step of a number below 1/2: 2^-26 turns, 2^-23 radians), the sine and cosine (4 steps, 2^-22), r
(a sum of 128 squares in a tree over 16-term chains, 20 steps at most, halved by the root, and the
root's 2) and the products (3 each) stay below 2^-18 of |n_i| + |n_{i+64}|.  The gradient's terms
have two such factors and a second sum of 128: 2^-17 of the sum of their magnitudes.  dw adds up
to T * heads terms in chains of at most 64 additions for the sizes here: 2^-16 of the sum of
magnitudes."""
import math

import numpy as np
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
D = 128
HALF = 2.0 ** -8


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


def make(T, hq, hk, seed, fused=True, start=0, base=1e6, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    H = hq + 2 * hk
    qkv = (torch.randn((T, H * D), generator=g) * scale).to(torch.bfloat16).to(DEV)
    q, k = qkv[:, :hq * D].unflatten(1, (hq, D)), qkv[:, hq * D:(hq + hk) * D].unflatten(1, (hk, D))
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(torch.bfloat16).to(DEV) for _ in range(2)]
    f = torch.from_numpy(base ** (-np.arange(0, D, 2) / D)).to(DEV)
    pos = (start + torch.randint(0, 5000, (T,), generator=g)).to(torch.int32).to(DEV)
    dy = [torch.randn((T, h, D), generator=g).to(torch.bfloat16).to(DEV) for h in (hq, hk)]
    return qkv, q, k, w, f, pos, dy


def wide(t):
    return t.detach().cpu().double()


def turn(x, f, pos, sign=1):
    """The rotation of [T][h][128] in 64 bits, and the size of the terms it adds."""
    a = sign * wide(pos)[:, None, None] * wide(f)
    lo, hi = x[..., :64], x[..., 64:]
    size = lo.abs() + hi.abs()
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1), \
        torch.cat([size, size], -1)


def formula(x, w, f, pos, eps):
    x, w = wide(x), wide(w)
    return turn(x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w, f, pos)


def formula_grad(dy, x, w, f, pos, eps):
    x, w = wide(x), wide(w)
    r = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    g, size = turn(wide(dy), f, pos, -1)
    u, us = g * w, size * w.abs()
    xn = x * r
    dx = r * (u - xn * (u * xn).mean(-1, keepdim=True))
    dxs = r * (us + xn.abs() * (us * xn.abs()).mean(-1, keepdim=True))
    return dx, dxs, g * xn, size * xn.abs()


def check(got, want, size, part, what):
    err = (wide(got) - want).abs()
    over = err - (HALF * want.abs() + part * size)
    assert bool((over <= 0).all()), (what, float(over.max()), float(err.max()))


SHAPES = [(1, 16, 8), (2, 1, 1), (7, 40, 8), (130, 5, 3), (33, 9, 17), (300, 32, 8), (64, 8, 1)]


@pytest.mark.parametrize("T,hq,hk", SHAPES)
@pytest.mark.parametrize("fused", [True, False])
def test_forward(T, hq, hk, fused):
    log(f"case rope T={T} heads={hq},{hk} fused={fused}")
    qkv, q, k, w, f, pos, _ = make(T, hq, hk, 10 * T + hq, fused)
    before = qkv.clone()
    qo, ko = S.qk_norm_rope(q, k, w[0], w[1], f, pos, 1e-6)
    for got, x, wt in ((qo, q, w[0]), (ko, k, w[1])):
        check(got, *formula(x, wt, f, pos, 1e-6), 2.0 ** -18, "forward")
    assert torch.equal(qkv.view(torch.int16), before.view(torch.int16))


@pytest.mark.parametrize("T,hq,hk", SHAPES)
def test_gradient(T, hq, hk):
    log(f"case rope gradient T={T} heads={hq},{hk}")
    _, q, k, w, f, pos, dy = make(T, hq, hk, 20 * T + hk)
    # both gradients inside one buffer of the fused projection's gradient
    buf = torch.full((T, (hq + 2 * hk) * D), 7.0, dtype=torch.bfloat16, device=DEV)
    dq, dk = (buf[:, :hq * D].unflatten(1, (hq, D)),
              buf[:, hq * D:(hq + hk) * D].unflatten(1, (hk, D)))
    out = S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos, 1e-6, dq=dq, dk=dk)
    assert out[0] is dq and out[1] is dk
    assert bool((buf[:, (hq + hk) * D:] == 7).all())
    for dx, dw, d, x, wt in ((dq, out[2], dy[0], q, w[0]), (dk, out[3], dy[1], k, w[1])):
        want, size, part, ps = formula_grad(d, x, wt, f, pos, 1e-6)
        check(dx, want, size, 2.0 ** -17, "dx")
        err = (wide(dw) - part.sum((0, 1))).abs()
        assert bool((err <= 2.0 ** -16 * ps.sum((0, 1))).all()), float(err.max())


def test_gradient_against_differences():
    # the loss sum(dy y) along random directions of q and of its weight, by central differences in
    # 64 bits (step h: truncation h^2 of third derivatives of order one, and 2^-52 / h)
    T, hq, hk, h = 9, 4, 2, 1e-4
    _, q, k, w, f, pos, dy = make(T, hq, hk, 5)
    dq, _, dwq, _ = S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos, 1e-6)
    g = torch.Generator().manual_seed(6)
    x, wt, d = wide(q), wide(w[0]), wide(dy[0])

    def loss(x, wt):
        n = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * wt
        return float((turn(n, f, pos)[0] * d).sum())
    for _ in range(5):
        e = torch.randn(x.shape, generator=g, dtype=torch.float64)
        want = (loss(x + h * e, wt) - loss(x - h * e, wt)) / (2 * h)
        tol = float(((HALF + 2.0 ** -15) * wide(dq).abs() * e.abs()).sum()) + 1e-3
        assert abs(float((wide(dq) * e).sum()) - want) <= tol
        e = torch.randn(D, generator=g, dtype=torch.float64)
        want = (loss(x, wt + h * e) - loss(x, wt - h * e)) / (2 * h)
        assert abs(float((wide(dwq) * e).sum()) - want) <= 1e-3 * max(1.0, abs(want))


def test_far_positions_and_other_frequencies():
    for start, base in ((131071, 1e6), (2 ** 31 - 1 - 5000, 1e4)):
        _, q, k, w, f, pos, _ = make(12, 3, 2, 8, start=start, base=base)
        pos[0] = 2 ** 31 - 1
        qo, ko = S.qk_norm_rope(q, k, w[0], w[1], f, pos, 1e-6)
        # (the reference's own angle is a product in 64 bits: 2^-53 of 2^31 radians)
        check(qo, *formula(q, w[0], f, pos, 1e-6), 2.0 ** -18, "far q")
        check(ko, *formula(k, w[1], f, pos, 1e-6), 2.0 ** -18, "far k")


@pytest.mark.parametrize("scale", [1e-20, 1e-3, 1e12])
def test_small_and_large_rows_and_zero_rows(scale):
    _, q, k, w, f, pos, dy = make(6, 4, 2, 9, fused=False, scale=scale)
    q[2] = 0
    qo, ko = S.qk_norm_rope(q, k, w[0], w[1], f, pos, 1e-6)
    check(qo, *formula(q, w[0], f, pos, 1e-6), 2.0 ** -18, "q")
    assert bool((qo[2] == 0).all())
    dq, dk, dwq, dwk = S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos, 1e-6)
    want, size, part, ps = formula_grad(dy[0], q, w[0], f, pos, 1e-6)
    check(dq, want, size, 2.0 ** -17, "dq")
    assert bool(torch.isfinite(dwq).all()) and bool(torch.isfinite(dwk).all())


def test_padding_rows():
    _, q, k, w, f, pos, dy = make(20, 5, 3, 11)
    pad = torch.tensor([0, 3, 4, 19], device=DEV)
    live = [i for i in range(20) if i not in (0, 3, 4, 19)]
    pos[pad] = -1
    qo = torch.full((20, 5, D), 3.0, dtype=torch.bfloat16, device=DEV)
    ko = torch.full((20, 3, D), 3.0, dtype=torch.bfloat16, device=DEV)
    S.qk_norm_rope(q, k, w[0], w[1], f, pos, 1e-6, q_out=qo, k_out=ko)
    assert bool((qo[pad] == 3).all()) and bool((ko[pad] == 3).all())
    want, size = formula(q, w[0], f, pos, 1e-6)
    check(qo[live], want[live], size[live], 2.0 ** -18, "live rows")
    # NaN in padding rows reaches nothing
    for t in (q, k, dy[0], dy[1]):
        t[pad] = float("nan")
    dq, dk, dwq, dwk = S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos, 1e-6)
    assert bool((dq[pad] == 0).all()) and bool((dk[pad] == 0).all())
    want, size, part, ps = formula_grad(dy[0][live], q[live], w[0], f, pos[live], 1e-6)
    check(dq[live], want, size, 2.0 ** -17, "live dq")
    assert bool(((wide(dwq) - part.sum((0, 1))).abs() <= 2.0 ** -16 * ps.sum((0, 1))).all())


def test_in_place():
    _, q, k, w, f, pos, dy = make(50, 6, 2, 12, fused=False)
    qo, ko = S.qk_norm_rope(q, k, w[0], w[1], f, pos)
    dq, dk, dwq, dwk = S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos)
    q2, k2 = q.clone(), k.clone()
    S.qk_norm_rope(q2, k2, w[0], w[1], f, pos, q_out=q2, k_out=k2)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)
    d0, d1 = dy[0].clone(), dy[1].clone()
    again = S.qk_norm_rope_bwd(d0, d1, q, k, w[0], w[1], f, pos, dq=d0, dk=d1)
    assert torch.equal(d0, dq) and torch.equal(d1, dk)
    assert torch.equal(again[2], dwq) and torch.equal(again[3], dwk)


def test_long_text_and_repeated_calls_are_equal():
    # more tokens than one round of the gradient's workgroups takes
    T, hq, hk = 9001, 4, 2
    _, q, k, w, f, pos, dy = make(T, hq, hk, 13)
    a = S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos)
    b = S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    want, size, part, ps = formula_grad(dy[0], q, w[0], f, pos, 1e-6)
    check(a[0], want, size, 2.0 ** -17, "dq")
    assert bool(((wide(a[2]) - part.sum((0, 1))).abs() <= 2.0 ** -16 * ps.sum((0, 1))).all())
    qo, _ = S.qk_norm_rope(q, k, w[0], w[1], f, pos)
    check(qo, *formula(q, w[0], f, pos, 1e-6), 2.0 ** -18, "long forward")


def test_no_tokens():
    _, q, k, w, f, pos, dy = make(0, 4, 2, 1)
    qo, ko = S.qk_norm_rope(q, k, w[0], w[1], f, pos)
    assert qo.shape == (0, 4, D) and ko.shape == (0, 2, D)
    dq, dk, dwq, dwk = S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos)
    assert dq.shape == (0, 4, D) and bool((dwq == 0).all()) and bool((dwk == 0).all())


def test_wrapper_refusals():
    _, q, k, w, f, pos, dy = make(6, 4, 2, 2)
    ok = dict(q=q, k=k, q_weight=w[0], k_weight=w[1], inv_freq=f, positions=pos)

    def bad(**kw):
        with pytest.raises((ValueError, RuntimeError)):
            S.qk_norm_rope(**(ok | kw))
        with pytest.raises((ValueError, RuntimeError)):
            S.qk_norm_rope_bwd(dy[0], dy[1], **(ok | kw))
    bad(q=q.float())
    bad(q=q[:, :, ::2])
    bad(q=q.transpose(0, 1).contiguous().transpose(0, 1))
    bad(k=k[:5])
    bad(q=q[..., :64])
    bad(q_weight=w[0].float())
    bad(k_weight=w[1][:64])
    bad(inv_freq=f.float())
    bad(positions=pos.long())
    bad(positions=pos[:5])
    bad(positions=pos.cpu())
    bad(eps=-1.0)
    with pytest.raises(ValueError):
        S.qk_norm_rope(**ok, q_out=torch.empty(6, 4, D, device=DEV))
    with pytest.raises(ValueError):
        S.qk_norm_rope_bwd(dy[0][:5], dy[1], **ok)
    with pytest.raises(S.SparrowError):
        S.qk_norm_rope_bwd(dy[0], dy[1], **ok, workspace=torch.empty(1024, dtype=torch.uint8,
                                                                     device=DEV))
    # an odd token stride breaks the 16-byte rows
    odd = torch.zeros(6, 4 * D + 4, dtype=torch.bfloat16, device=DEV)[:, :4 * D].unflatten(1, (4, D))
    bad(q=odd)


def test_side_stream_and_graph_replays():
    T, hq, hk = 77, 8, 2
    _, q, k, w, f, pos, dy = make(T, hq, hk, 14, fused=False)
    want = S.qk_norm_rope(q, k, w[0], w[1], f, pos)
    wg = S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    ws = torch.empty(S.SPARROW_ROPE_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    outs = [torch.zeros_like(t) for t in want + wg]
    with torch.cuda.stream(side):
        a = S.qk_norm_rope(q, k, w[0], w[1], f, pos)
        assert all(torch.equal(x, y) for x, y in zip(a, want))
        with torch.cuda.graph(graph, stream=side):
            S.qk_norm_rope(q, k, w[0], w[1], f, pos, q_out=outs[0], k_out=outs[1])
            S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos, dq=outs[2], dk=outs[3],
                               dq_weight=outs[4], dk_weight=outs[5], workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(3):
        for o in outs:
            o.fill_(math.nan)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want + wg)), rep


@pytest.mark.parametrize("T,hq,hk", [(1, 1024, 1024), (5, 1000, 3), (700, 3, 1000)])
def test_many_heads(T, hq, hk):
    log(f"case rope many heads T={T} heads={hq},{hk}")
    _, q, k, w, f, pos, dy = make(T, hq, hk, 30 + T)
    got = S.qk_norm_rope(q, k, w[0], w[1], f, pos)
    out = S.qk_norm_rope_bwd(dy[0], dy[1], q, k, w[0], w[1], f, pos)
    for i, (x, wt) in enumerate(((q, w[0]), (k, w[1]))):
        check(got[i], *formula(x, wt, f, pos, 1e-6), 2.0 ** -18, "forward")
        want, size, part, ps = formula_grad(dy[i], x, wt, f, pos, 1e-6)
        check(out[i], want, size, 2.0 ** -17, "dx")
        # (at most 700,000 rows over some 2000 waves of 8 rows a pass: 44 additions a lane)
        assert bool(((wide(out[2 + i]) - part.sum((0, 1))).abs() <= 2.0 ** -16 * ps.sum((0, 1))).all())


def test_offsets_past_32_bits():
    # 2.3e9 elements of q and of its gradient, streamed stores; the last tokens against the formula,
    # and rows of padding in front of them as they were
    T, hq, hk, n = 70000, 256, 1, 40
    f = torch.from_numpy(1e6 ** (-np.arange(0, D, 2) / D)).to(DEV)
    w = [torch.full((D,), 1.25, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    pos[T - n - 3:T - n] = -1
    g = torch.Generator(device=DEV).manual_seed(31)
    q, k, dq_out, dk_out = (torch.randn((T, h, D), generator=g, device=DEV, dtype=torch.bfloat16)
                            for h in (hq, hk, hq, hk))
    outs = [torch.full_like(t, 7.0) for t in (q, k)]
    S.qk_norm_rope(q, k, w[0], w[1], f, pos, q_out=outs[0], k_out=outs[1])
    grads = S.qk_norm_rope_bwd(dq_out, dk_out, q, k, w[0], w[1], f, pos)
    for i, (x, dy) in enumerate(((q, dq_out), (k, dk_out))):
        check(outs[i][-n:], *formula(x[-n:], w[i], f, pos[-n:], 1e-6), 2.0 ** -18, "far rows")
        check(grads[i][-n:], *formula_grad(dy[-n:], x[-n:], w[i], f, pos[-n:], 1e-6)[:2],
              2.0 ** -17, "far dx")
        assert bool((outs[i][T - n - 3:T - n] == 7).all())
        assert bool((grads[i][T - n - 3:T - n] == 0).all())
