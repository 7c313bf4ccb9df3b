"""Token sampling where zeros of either sign are the largest logits, against the definition in 64 bits: -0 equals +0."""
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log
from test_gpu_sample import check, ints, rand

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


def filters(T, V, seed):
    """Top-k below and above what is sorted, top-p, both, all three."""
    few, many = ints(T, seed, 2, 60), ints(T, seed + 1, min(1100, V - 1), V - 1)
    p, q = rand(T, seed + 2, 0.1, 0.99), rand(T, seed + 3, 1e-4, 0.5)
    return [dict(), dict(k=few), dict(k=many), dict(p=p), dict(q=q), dict(k=few, p=p), dict(k=many, p=p),
            dict(k=many, p=p, q=q)]


@pytest.mark.parametrize("V", [1030, 5000, 60013])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_rows_of_negative_zeros(V, dtype):
    # all tokens are equal: the borders of the filters are whole numbers of them
    log(f"case sample all -0 V={V} {dtype}")
    T = 8
    z = torch.full((T, V), -0.0, dtype=dtype, device=DEV)
    for kw in filters(T, V, V):
        check(z, torch.tensor([0.0, 0.25, 0.5, 0.75] * 2, device=DEV), **kw)


@pytest.mark.parametrize("V", [1030, 5000, 60013])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("top", ["half", "one", "both signs", "mask"])
def test_negative_zero_is_the_largest(V, dtype, top):
    log(f"case sample largest -0 {top} V={V} {dtype}")
    T = 12
    g = torch.Generator().manual_seed(V + len(top))
    z = -torch.randn((T, V), generator=g).abs() - 0.01
    if top == "one":
        z[torch.arange(T), torch.randint(0, V, (T,), generator=g)] = -0.0
    else:
        z[torch.rand((T, V), generator=g) < 0.5] = -0.0
    if top == "both signs":
        z[(z == 0) & (torch.rand((T, V), generator=g) < 0.3)] = 0.0
    if top == "mask":                       # -(1 - allowed) * 1e9
        z = -(1 - (z == 0).float()) * 1e9
    z = z.to(dtype).to(DEV)
    for kw in filters(T, V, V):
        check(z, rand(T, V), **kw)
        check(z, rand(T, V + 1), t=rand(T, V + 2, 0.5, 2.0), **kw)
