"""Operators that are no autograd node refuse inputs that a gradient is recorded for, or that carry a forward-mode
tangent, which they would drop; and take the same ones where none is recorded."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2606_08446_amd import sparrow as S

BF = torch.bfloat16


def rope(dev):
    x = [torch.zeros((3, 2, 128), dtype=BF, device=dev) for _ in range(2)]
    w = [torch.ones(128, dtype=BF, device=dev) for _ in range(2)]
    f = torch.zeros(64, dtype=torch.float64, device=dev)
    return x + w, lambda *a: S.qk_norm_rope(*a, f, torch.arange(3, dtype=torch.int32, device=dev))


def norm(dev):
    z, w = torch.ones((3, 64), dtype=BF, device=dev), torch.ones(64, dtype=BF, device=dev)
    return [z, z.clone(), w, w.clone(), z.clone()], S.residual_norm


def norm_bwd(dev):
    z, w = torch.ones((3, 64), dtype=BF, device=dev), torch.ones(64, dtype=BF, device=dev)
    return [z, z.clone(), z.clone(), z.clone(), w, w.clone(), z.clone()], S.residual_norm_bwd


def shared(dev):
    i = dict(dtype=torch.int32, device=dev)
    c = [torch.ones((4, 1, 16, 128), dtype=BF, device=dev) for _ in range(2)]
    rest = (torch.arange(4, **i).view(2, 2), torch.full((2,), 20, **i), torch.tensor([0, 2], **i),
            torch.full((1,), 16, **i))
    return [torch.ones((2, 2, 128), dtype=BF, device=dev)] + c, \
        lambda q, k, v: S.shared_prefix_decode_attn(q, k, v, *rest)


def sample(dev):
    one = torch.full((2,), 0.5, device=dev)
    return [torch.zeros((2, 9), device=dev)] + [one.clone() for _ in range(4)], \
        lambda z, u, t, p, q: S.sample(z, u, t, None, p, q)


OPERATORS = [(f, i) for f, n in ((rope, 4), (norm, 5), (norm_bwd, 7), (shared, 3), (sample, 5)) for i in range(n)]


@pytest.mark.parametrize("make,i", OPERATORS)
def test_refusals(make, i):
    a, call = make("cpu")
    a[i].requires_grad_()
    with pytest.raises(ValueError, match="records no gradient"):
        call(*a)
    with torch.no_grad(), pytest.raises(RuntimeError, match="GPU"):     # (goes on to the next check)
        call(*a)
    a[i].requires_grad_(False)
    with forward_ad.dual_level():
        b = list(a)
        b[i] = forward_ad.make_dual(a[i], torch.ones_like(a[i]))
        with pytest.raises(ValueError, match="records no gradient"):
            call(*b)
        with pytest.raises(RuntimeError, match="GPU"):
            call(*a)


def flat(x):
    return [t for t in (x if isinstance(x, tuple) else (x,)) if t is not None]


@pytest.mark.gpu
@pytest.mark.parametrize("make", [rope, norm, norm_bwd, shared, sample])
def test_the_same_inputs_without_a_gradient(gpu_device, make):
    a, call = make("cuda")
    want = flat(call(*a))
    for t in a:
        t.requires_grad_()
    with pytest.raises(ValueError, match="records no gradient"):
        call(*a)
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            got = flat(call(*a))
        assert all(torch.equal(x, y) and not x.requires_grad for x, y in zip(got, want))
