"""The head norms' wrapper refuses inputs that autograd records a gradient for, which it would drop, and
takes the same ones where none is recorded."""
import pytest
import torch

from paper_2606_08446_amd import sparrow as S


def inputs(device):
    g = torch.Generator().manual_seed(0)
    q, k = (torch.randn((5, h, 128), generator=g).to(torch.bfloat16).to(device) for h in (4, 2))
    w = [torch.ones(128, dtype=torch.bfloat16, device=device) for _ in range(2)]
    f = torch.linspace(0.0, 1.0, 64, dtype=torch.float64, device=device)
    return [q, k, *w, f, torch.arange(5, dtype=torch.int32, device=device)]


@pytest.mark.parametrize("i", range(4))
def test_recorded_gradients_are_refused(i):
    a = inputs("cpu")
    a[i].requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        S.qk_norm_rope(*a)
    with torch.no_grad(), pytest.raises(RuntimeError, match="GPU"):     # (goes on to the next check)
        S.qk_norm_rope(*a)


@pytest.mark.gpu
def test_leaves_without_a_recorded_gradient(gpu_device):
    a = inputs("cuda")
    want = S.qk_norm_rope(*a)
    for t in a[:4]:
        t.requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        S.qk_norm_rope(*a)
    with torch.no_grad():
        got = S.qk_norm_rope(*a)
    assert all(torch.equal(x, y) and not x.requires_grad for x, y in zip(got, want))
    grads = S.qk_norm_rope_bwd(*got, *a)                                # (a plain function of its own)
    assert not any(t.requires_grad for t in grads)

    class Node(torch.autograd.Function):                                # as a trainer's own node calls it
        @staticmethod
        def forward(ctx, *x):
            ctx.save_for_backward(*x)
            return S.qk_norm_rope(*x)

        @staticmethod
        def backward(ctx, dq, dk):
            dq, dk, dwq, dwk = S.qk_norm_rope_bwd(dq, dk, *ctx.saved_tensors)
            return dq, dk, dwq.to(torch.bfloat16), dwk.to(torch.bfloat16), None, None
    torch.autograd.backward(Node.apply(*a), got)
    for t, d in zip(a[:4], grads):
        assert torch.equal(t.grad, d.to(torch.bfloat16))
