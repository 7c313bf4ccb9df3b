"""The norms around a block and their gradient against the formulas in 64 bits (on the CPU).

Tolerances.  One rounding to bf16 is off by at most 2^-8 of the value here, to fp32 by 2^-24.  In fp32, a
sum over a row is a chain of at most 16 terms a thread, a scan of 6 steps and a chain of 16 waves: 40
steps of 2^-24 of the sum of magnitudes, and r half of that with the root's own 2: 2^-19.  b = scale
sigmoid(gate) x r_x post_weight has r_x, a sigmoid (6) and 5 products: 2^-18.4 of |b|; y has b's error,
an addition, r's error (r moves with h' too: y |h'| (|h| + |b|) over the row's mean square) and 3
products: 2^-18 of the terms' magnitudes.  The gradient's terms go through two such sums one after the
other: 2^-17 for dh, 2^-16 behind it.  The weights' sums are chains over the tokens of a workgroup, then of
at most 64 workgroups, then 32: under 150 steps at the sizes here on top of the terms' errors, 2^-15.
A sigmoid below fp32's smallest normal number, 2^-126, may become 0: with factors of at most 64 on it
(a gradient of the order of 1, r_x, weights) that is 2^-120."""
import math

import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16 = 2.0 ** -8
TINY = 2.0 ** -120
STEP = {torch.bfloat16: BF16, torch.float32: 2.0 ** -24}


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


def make(T, C, seed, post=True, gate=True, stream=torch.bfloat16, fused=True, scale=0.3, big=1.0):
    g = torch.Generator().manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=g)
    xg = (randn(T, 2 * C) * big).to(torch.bfloat16).to(DEV)
    x, a = xg[:, :C], xg[:, C:]
    if not fused:
        x, a = x.contiguous(), a.contiguous()
    d = dict(h=(randn(T, C) * 2 * big).to(stream).to(DEV), x=x, gate=a if gate else None,
             weight=(1 + 0.3 * randn(C)).to(torch.bfloat16).to(DEV),
             post_weight=(1 + 0.3 * randn(C)).to(torch.bfloat16).to(DEV) if post else None,
             scale=scale, eps=1e-6)
    dy = randn(T, C).to(torch.bfloat16).to(DEV)
    dh = randn(T, C).to(stream).to(DEV)
    return d, dy, dh


def wide(t):
    return t.detach().cpu().double()


def formula(h, x, weight, post_weight, gate, scale, eps):
    """(h', its size, y, its size) in 64 bits."""
    h, w = wide(h), wide(weight)
    b = torch.zeros_like(h)
    if x is not None:
        b = scale * wide(x)
        if post_weight is not None:
            b = b / (wide(x).square().mean(-1, keepdim=True) + eps).sqrt() * wide(post_weight)
        if gate is not None:
            b = b * torch.sigmoid(wide(gate))
    hp, size = h + b, h.abs() + b.abs()
    ms = hp.square().mean(-1, keepdim=True) + eps
    y = hp / ms.sqrt() * w
    move = (size * hp.abs()).mean(-1, keepdim=True) / ms
    return hp, size, y, w.abs() / ms.sqrt() * (size + hp.abs() * (1 + move))


def formula_grad(dy, dh_out, h, x, weight, post_weight, gate, scale, eps):
    """name -> (gradient, sum of its terms' magnitudes), per token for the weights."""
    h, w, dy = wide(h), wide(weight), wide(dy)
    r = 1 / (h.square().mean(-1, keepdim=True) + eps).sqrt()
    k, u = h * r, dy * w
    dh = r * (u - k * (u * k).mean(-1, keepdim=True))
    dhs = r * (u.abs() + 2 * k.abs() * (u * k).abs().mean(-1, keepdim=True))
    if dh_out is not None:
        dh, dhs = dh + wide(dh_out), dhs + wide(dh_out).abs()
    out = dict(dh=(dh, dhs), dweight=(dy * k, (dy * k).abs()))
    d, ds = scale * dh, abs(scale) * dhs
    if x is None:
        return out
    x = wide(x)
    kx, rx = x, 1.0
    if post_weight is not None:
        rx = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
        kx = x * rx
    p = 1.0 if post_weight is None else wide(post_weight)
    if gate is not None:
        s = torch.sigmoid(wide(gate))
        q = kx * p * s * torch.sigmoid(-wide(gate))  # (1 - s: near s = 1 that loses 64 bits' digits too)
        out["dgate"] = (d * q, ds * q.abs())
        d, ds = d * s, ds * s
    if post_weight is not None:
        out["dpost_weight"] = (d * kx, ds * kx.abs())
        v, vs = d * p, ds * p.abs()
        d = rx * (v - kx * (v * kx).mean(-1, keepdim=True))
        ds = rx * (vs + 2 * kx.abs() * (vs * kx.abs()).mean(-1, keepdim=True))
    out["dx"] = (d, ds)
    return out


def close(got, want, step, part, size, what):
    over = (wide(got) - want).abs() - (step * want.abs() + part * size + TINY)
    assert bool((over <= 0).all()), (what, float(over.max()))


def check_forward(d, got):
    hp, hs, y, ys = formula(**d)
    if d["x"] is not None:
        close(got[0], hp, STEP[got[0].dtype], 2.0 ** -18, hs, "h")
    close(got[1], y, BF16, 2.0 ** -18, ys, "y")


def check_backward(d, dy, dh, got, chain=2.0 ** -15):
    want = formula_grad(dy, dh, **d)
    names = ("dh", "dx", "dgate", "dweight", "dpost_weight")
    assert {n for n, t in zip(names, got) if t is not None} == set(want)
    for name, t in zip(names, got):
        if name in ("dweight", "dpost_weight") and t is not None:
            val, size = want[name]
            err = (wide(t) - val.sum(0)).abs()
            assert t.dtype == torch.float32
            assert bool((err <= chain * size.sum(0)).all()), (name, float((err / size.sum(0)).max()))
        elif t is not None:
            close(t, want[name][0], STEP[t.dtype], 2.0 ** -17 if name == "dh" else 2.0 ** -16,
                  want[name][1], name)


SHAPES = [(1, 8), (1, 2048), (2, 16384), (3, 8200), (5, 8192), (37, 264), (130, 4096), (61, 5120),
          (33, 504), (2100, 128)]


@pytest.mark.parametrize("T,C", SHAPES)
@pytest.mark.parametrize("post,gate", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32])
def test_both_directions(T, C, post, gate, stream):
    log(f"case residual_norm T={T} C={C} post={post} gate={gate} {stream}")
    d, dy, dh = make(T, C, T + C, post, gate, stream, fused=T % 2 == 1)
    check_forward(d, S.residual_norm(**d))
    d["h"] = S.residual_norm(**d)[0]
    e = dict(d, h_out=d["h"])
    del e["h"]
    check_backward(d, dy, dh, S.residual_norm_bwd(dy, dh, **e))


def grad(dy, dh_out, d, **kw):
    return S.residual_norm_bwd(dy, dh_out, d["h"], d["x"], d["weight"], d["post_weight"], d["gate"],
                               d["scale"], d["eps"], **kw)


def test_first_norm_and_last_gradient():
    # no block in front, and nothing behind that a gradient comes from
    for stream in (torch.bfloat16, torch.float32):
        d, dy, dh = make(19, 640, 3, post=False, gate=False, stream=stream)
        d["x"] = None
        h, y = S.residual_norm(**d)
        assert h is d["h"]
        check_forward(d, (h, y))
        check_backward(d, dy, None, grad(dy, None, d, block=False))
        check_backward(d, dy, dh, grad(dy, dh, d, block=False))


def test_the_block_alone_is_not_needed_without_norm_and_gate():
    d, dy, dh = make(19, 640, 4, post=False, gate=False)
    a, b = grad(dy, dh, d), grad(dy, dh, d | dict(x=None))
    assert all(torch.equal(s, t) for s, t in zip(a, b) if s is not None)


def test_gradient_against_differences():
    # the loss sum(dy y) + sum(dh h') along random directions, by central differences in 64 bits (step
    # e: truncation e^2 of third derivatives of order one, and 2^-52 / e)
    T, C, e = 6, 64, 1e-4
    d, dy, dh = make(T, C, 5, stream=torch.float32)
    hp = S.residual_norm(**d)[0]
    got = dict(zip(("h", "x", "gate", "weight", "post_weight"),
                   grad(dy, dh, d | dict(h=hp))))
    g = torch.Generator().manual_seed(6)
    wdy, wdh = wide(dy), wide(dh)

    def loss(kw):
        h, _, y, _ = formula(**kw)
        return float((y * wdy).sum() + (h * wdh).sum())
    for name, t in got.items():
        for _ in range(3):
            move = torch.randn(t.shape, generator=g, dtype=torch.float64)
            at = {k: (v.cpu().double() if isinstance(v, torch.Tensor) else v) for k, v in d.items()}
            hi, lo = dict(at), dict(at)
            hi[name], lo[name] = at[name] + e * move, at[name] - e * move
            want = (loss(hi) - loss(lo)) / (2 * e)
            tol = float(((BF16 + 2.0 ** -14) * wide(t).abs() * move.abs()).sum()) + 1e-4
            assert abs(float((wide(t) * move).sum()) - want) <= tol, name


@pytest.mark.parametrize("big", [1e-20, 1e-3, 1e12])
def test_small_and_large_rows_and_zero_rows(big):
    d, dy, dh = make(7, 1000, 9, gate=False, big=big)
    d["h"][2] = 0
    d["x"][2] = 0
    h, y = S.residual_norm(**d)
    check_forward(d, (h, y))
    assert bool((h[2] == 0).all()) and bool((y[2] == 0).all())
    out = grad(dy, dh, d)
    assert all(bool(torch.isfinite(t).all()) for t in out if t is not None)
    if big >= 1e-3:
        check_backward(d, dy, dh, out)


def test_far_gates():
    # a closed gate lets nothing through, an open one everything, and neither is steep
    d, dy, dh = make(4, 256, 10, post=False)
    d["gate"] = d["gate"].clone()
    for i, v in enumerate((-200.0, 200.0, -30.0, 30.0)):
        d["gate"][i] = v
    check_forward(d, S.residual_norm(**d))
    out = grad(dy, dh, d)
    check_backward(d, dy, dh, out)
    assert bool((out[1][0] == 0).all()) and bool((out[2][:2] == 0).all())


def test_rows_do_not_touch_each_other():
    d, dy, dh = make(12, 512, 11, fused=False)
    want, wg = S.residual_norm(**d), grad(dy, dh, d)
    for name in ("h", "x", "gate"):
        d[name][5] = math.nan
    got, gg = S.residual_norm(**d), grad(dy, dh, d)
    keep = [i for i in range(12) if i != 5]
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip(want, got))
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip(wg[:3], gg[:3]))
    assert bool(got[1][5].isnan().all())


def test_in_place_and_views():
    T, C = 50, 768
    d, dy, dh = make(T, C, 12)
    want, wg = S.residual_norm(**d), grad(dy, dh, d)
    h = d["h"].clone()
    got = S.residual_norm(**(d | dict(h=h)), h_out=h)
    assert got[0] is h and torch.equal(h, want[0]) and torch.equal(got[1], want[1])
    buf = torch.full((T, 3 * C), 7.0, dtype=torch.bfloat16, device=DEV)
    dh2 = dh.clone()
    out = grad(dy, dh2, d, dh=dh2, dx=buf[:, :C], dgate=buf[:, 2 * C:])
    assert out[0] is dh2 and all(torch.equal(a, b) for a, b in zip(out, wg))
    assert bool((buf[:, C:2 * C] == 7).all())


def test_many_tokens_and_repeated_calls_are_equal():
    T, C = 9001, 256
    d, dy, dh = make(T, C, 13)
    a, b = grad(dy, dh, d), grad(dy, dh, d)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    check_backward(d, dy, dh, a)
    check_forward(d, S.residual_norm(**d))


def test_no_tokens():
    d, dy, dh = make(0, 64, 1)
    h, y = S.residual_norm(**d)
    assert h.shape == y.shape == (0, 64)
    out = grad(dy, dh, d)
    assert out[0].shape == (0, 64) and bool((out[3] == 0).all()) and bool((out[4] == 0).all())


def test_wrapper_refusals():
    d, dy, dh = make(6, 64, 2)

    def bad(**kw):
        with pytest.raises((ValueError, RuntimeError)):
            S.residual_norm(**(d | kw))
        with pytest.raises((ValueError, RuntimeError)):
            grad(dy, dh, d | kw)
    bad(h=d["h"].half())
    bad(h=d["h"][:, ::2])
    bad(h=d["h"][:5])
    bad(h=d["h"][0])
    bad(h=d["h"].cpu())
    bad(x=d["x"].float())
    bad(x=d["x"][:5])
    bad(x=d["x"].t().contiguous().t())
    bad(x=torch.zeros(6, 68, dtype=torch.bfloat16, device=DEV)[:, :64])
    bad(x=d["x"][:1].expand(6, 64))
    bad(x=None)
    bad(gate=d["gate"].float())
    bad(weight=d["weight"].float())
    bad(weight=d["weight"][:32])
    bad(post_weight=d["post_weight"].cpu())
    bad(eps=-1.0)
    bad(scale=math.inf)
    with pytest.raises(ValueError):
        S.residual_norm(**d, h_out=torch.empty(6, 64, device=DEV))
    with pytest.raises(ValueError):
        grad(dy[:5], dh, d)
    with pytest.raises(ValueError):
        grad(dy, dh.float(), d)
    with pytest.raises(ValueError):
        grad(dy, dh, d | dict(gate=None), dgate=dy)
    with pytest.raises(S.SparrowError):
        grad(dy, dh, d, workspace=torch.empty(64, dtype=torch.uint8, device=DEV))


def test_side_stream_and_graph_replays():
    d, dy, dh = make(77, 2056, 14, fused=False)
    want, wg = S.residual_norm(**d), grad(dy, dh, d)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    ws = torch.empty(S.sparrow_residual_norm_workspace_size(77, 2056), dtype=torch.uint8, device=DEV)
    outs = [torch.zeros_like(t) for t in want + wg]
    with torch.cuda.stream(side):
        a = S.residual_norm(**d)
        assert all(torch.equal(x, y) for x, y in zip(a, want))
        with torch.cuda.graph(graph, stream=side):
            S.residual_norm(**d, h_out=outs[0], y=outs[1])
            grad(dy, dh, d, dh=outs[2], dx=outs[3], dgate=outs[4], dweight=outs[5],
                 dpost_weight=outs[6], workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(3):
        for o in outs:
            o.fill_(math.nan)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want + wg)), rep


@pytest.mark.parametrize("C", [1040, 2056, 4104, 8200, 16264])
@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32])
def test_gradient_in_place(C, stream):
    # dh over dh_out, where threads and whole waves lie past the row's end
    log(f"case residual_norm_bwd in place C={C} {stream}")
    d, dy, dh = make(1500, C, C, stream=stream, fused=False)
    want = grad(dy, dh, d)
    got = grad(dy, dh, d, dh=dh)
    assert got[0].data_ptr() == dh.data_ptr()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_a_trainers_node():
    d, dy, dh = make(9, 128, 15, stream=torch.float32)
    leaves = [d[n] for n in ("h", "x", "weight", "post_weight", "gate")]
    leaves[1], leaves[4] = leaves[1].clone(), leaves[4].clone()
    want = S.residual_norm(*leaves, scale=0.3)
    for t in leaves:
        t.requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        S.residual_norm(*leaves, scale=0.3)

    class Node(torch.autograd.Function):
        @staticmethod
        def forward(ctx, h, x, w, p, a):
            hp, y = S.residual_norm(h, x, w, p, a, scale=0.3)
            ctx.save_for_backward(hp, x, w, p, a)
            return hp, y

        @staticmethod
        def backward(ctx, dh, dy):
            hp, x, w, p, a = ctx.saved_tensors
            g = S.residual_norm_bwd(dy, dh, hp, x, w, p, a, scale=0.3)
            return g[0], g[1], g[3].to(torch.bfloat16), g[4].to(torch.bfloat16), g[2]
    torch.autograd.backward(Node.apply(*leaves), (dh, dy))
    g = S.residual_norm_bwd(dy, dh, want[0], *(t.detach() for t in leaves[1:]), scale=0.3)
    for t, v in zip(leaves, (g[0], g[1], g[3], g[4], g[2])):
        assert torch.equal(t.grad, v.to(t.dtype))


def test_offsets_past_32_bits():
    # 2.2e9 elements of every array; the last tokens against the formula
    T, C, n = 2200000, 1000, 30
    g = torch.Generator(device=DEV).manual_seed(31)
    h, x, dy, dh = (torch.randn((T, C), generator=g, device=DEV, dtype=torch.bfloat16)
                    for _ in range(4))
    w, p = (torch.full((C,), 1.25, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    d = dict(h=h, x=x, weight=w, post_weight=p, gate=None, scale=0.5, eps=1e-6)
    end = d | dict(h=h[-n:], x=x[-n:])
    got = S.residual_norm(**d)
    check_forward(end, [t[-n:] for t in got])
    out = grad(dy, dh, d)
    want = formula_grad(dy[-n:], dh[-n:], **end)
    close(out[0][-n:], want["dh"][0], BF16, 2.0 ** -17, want["dh"][1], "dh")
    close(out[1][-n:], want["dx"][0], BF16, 2.0 ** -16, want["dx"][1], "dx")
    assert all(bool(torch.isfinite(t).all()) for t in out[3:])
