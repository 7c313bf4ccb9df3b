"""Offsets beyond 32 bits in attention over shared prefixes, token sampling and the norms around a block: rows and
pages far into large buffers against the same values in small ones, bit for bit (an operator's result depends
on its own rows and the sizes that its work is split by, which are the same)."""
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF = torch.bfloat16
BIG = 1 << 32


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield
    torch.cuda.empty_cache()


def test_pages_far_into_the_cache():
    hq, hkv, ps, D = 8, 2, 32, 128
    P = BIG // (hkv * ps * D) + 40
    log(f"case shared long pages={P}")
    lens = torch.tensor([200, 230, 190, 77], dtype=torch.int32, device=DEV)
    cu = torch.tensor([0, 3, 4], dtype=torch.int32, device=DEV)
    prefix = torch.tensor([150, 64], dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(1)
    q = torch.randn((4, hq, D), generator=g).to(BF).to(DEV)
    small = [torch.randn((40, hkv, ps, D), generator=g).to(BF).to(DEV) for _ in range(2)]
    table = torch.randperm(40, generator=g)[:32].view(4, 8).to(torch.int32).to(DEV)
    want = S.shared_prefix_decode_attn(q, *small, table, lens, cu, prefix)
    large = [torch.empty((P, hkv, ps, D), dtype=BF, device=DEV) for _ in range(2)]
    for a, b in zip(large, small):
        a[P - 40:] = b
    got = S.shared_prefix_decode_attn(q, *large, table + (P - 40), lens, cu, prefix)
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.float32, BF])
def test_logit_rows_far_apart(dtype):
    V, T, stride = 50021, 5, (1 << 30) + 12345
    log(f"case sample long stride={stride} {dtype}")
    g = torch.Generator().manual_seed(2)
    z = (3 * torch.randn((T, V), generator=g)).to(dtype).to(DEV)
    u, p = torch.rand(T, generator=g).to(DEV), torch.full((T,), 0.9, device=DEV)
    k = torch.tensor([0, 20, 0, 3, 0], dtype=torch.int32, device=DEV)
    far = torch.empty((T - 1) * stride + V, dtype=dtype, device=DEV).as_strided((T, V), (stride, 1))
    far.copy_(z)
    for kw in (dict(), dict(top_k=k, top_p=p), dict(top_p=p)):
        for a, b in zip(S.sample(far, u, **kw), S.sample(z, u, **kw)):
            assert torch.equal(a, b)


def test_more_rows_than_a_grid_has():
    T, V = 70001, 37
    log("case sample many rows")
    g = torch.Generator().manual_seed(3)
    z, u = torch.randn((T, V), generator=g).to(DEV), torch.rand(T, generator=g).to(DEV)
    p = torch.full((T,), 0.8, device=DEV)
    tail = slice(T - 5000, T)
    for kw, part in ((dict(), dict()), (dict(top_p=p), dict(top_p=p[tail]))):
        for a, b in zip(S.sample(z, u, **kw), S.sample(z[tail], u[tail], **part)):
            assert torch.equal(a[tail], b)


def test_norms_of_large_arrays():
    C = 16384
    T = BIG // C + 300
    log(f"case residual_norm long T={T} C={C}")
    g = torch.Generator(device=DEV).manual_seed(4)

    def randn(*shape):
        return torch.empty(shape, dtype=BF, device=DEV).normal_(generator=g)
    h, x, gate, dy, dh = (randn(T, C) for _ in range(5))
    w, post = randn(C), randn(C)
    hp, y = S.residual_norm(h, x, w, post, gate, 0.5)
    tail = slice(T - 200, T)
    a, b = S.residual_norm(h[tail].clone(), x[tail], w, post, gate[tail], 0.5)
    assert torch.equal(hp[tail], a) and torch.equal(y[tail], b)
    del y, b
    got = S.residual_norm_bwd(dy, dh, hp, x, w, post, gate, 0.5)
    want = S.residual_norm_bwd(dy[tail].clone(), dh[tail].clone(), a, x[tail], w, post, gate[tail], 0.5)
    for i in range(3):
        assert torch.equal(got[i][tail], want[i])
    assert all(bool(torch.isfinite(t).all()) for t in got[3:])
