"""sparrow_residual_norm and its gradient refuse bad host-visible arguments before any launch."""
import pytest

from paper_2606_08446_amd import sparrow as S

FAKE = 0x1000
BAD = [(dict(T=-1), S.SPARROW_EINVAL), (dict(T=1 << 31), S.SPARROW_EINVAL),
       (dict(C=0), S.SPARROW_EINVAL), (dict(C=-8), S.SPARROW_EINVAL),
       (dict(C=252), S.SPARROW_EUNSUPPORTED),
       (dict(C=16392, xs=16392, gs=16392, dxs=16392, dgs=16392), S.SPARROW_EUNSUPPORTED),
       (dict(dt=2), S.SPARROW_EUNSUPPORTED), (dict(dt=-1), S.SPARROW_EUNSUPPORTED),
       (dict(xs=248), S.SPARROW_EINVAL), (dict(xs=260), S.SPARROW_EINVAL),
       (dict(gs=248), S.SPARROW_EINVAL), (dict(gs=-512), S.SPARROW_EINVAL),
       (dict(eps=-1e-6), S.SPARROW_EINVAL), (dict(eps=float("nan")), S.SPARROW_EINVAL),
       (dict(scale=float("inf")), S.SPARROW_EINVAL), (dict(scale=float("nan")), S.SPARROW_EINVAL)]


def forward(**kw):
    a = dict(T=3, C=256, dt=1, h=FAKE, x=FAKE, xs=512, g=FAKE, gs=512, w=FAKE, p=FAKE, scale=1.0,
             eps=1e-6, ho=FAKE, y=FAKE) | kw
    return S.sparrow_residual_norm(a["T"], a["C"], a["dt"], a["h"], a["x"], a["xs"], a["g"], a["gs"],
                                   a["w"], a["p"], a["scale"], a["eps"], a["ho"], a["y"], None)


def backward(**kw):
    a = dict(T=3, C=256, dt=1, dy=FAKE, dho=FAKE, h=FAKE, x=FAKE, xs=512, g=FAKE, gs=512, w=FAKE,
             p=FAKE, scale=1.0, eps=1e-6, dh=FAKE, dx=FAKE, dxs=512, dg=FAKE, dgs=512, dw=FAKE,
             dp=FAKE, ws=FAKE, n=1 << 40) | kw
    return S.sparrow_residual_norm_bwd(
        a["T"], a["C"], a["dt"], a["dy"], a["dho"], a["h"], a["x"], a["xs"], a["g"], a["gs"], a["w"],
        a["p"], a["scale"], a["eps"], a["dh"], a["dx"], a["dxs"], a["dg"], a["dgs"], a["dw"],
        a["dp"], a["ws"], a["n"], None)


@pytest.mark.parametrize("bad,status", BAD)
def test_bad_sizes_are_refused(bad, status):
    assert forward(**{k: v for k, v in bad.items() if k not in ("dxs", "dgs")}) == status
    assert backward(**bad) == status


@pytest.mark.parametrize("name", ["h", "x", "w", "ho", "y"])
def test_forward_pointers(name):
    assert forward(**{name: None}) == S.SPARROW_EINVAL


@pytest.mark.parametrize("name", ["h", "x", "g", "w", "p", "ho", "y"])
def test_forward_alignment(name):
    assert forward(**{name: FAKE + 8}) == S.SPARROW_EINVAL


def test_nothing_goes_without_the_block():
    for name in ("g", "p", "ho"):
        alone = dict(x=None, g=None, p=None, ho=None) | {name: FAKE}
        assert forward(**alone) == S.SPARROW_EINVAL


@pytest.mark.parametrize("name", ["dy", "h", "x", "g", "w", "p", "dh", "dx", "dg", "dw", "dp"])
def test_backward_pointers(name):
    assert backward(**{name: None}) == S.SPARROW_EINVAL
    assert backward(**{name: FAKE + 2}) == S.SPARROW_EINVAL


def test_backward_strides_and_workspace():
    assert backward(dho=FAKE + 8) == S.SPARROW_EINVAL
    assert backward(dxs=248) == S.SPARROW_EINVAL
    assert backward(dgs=260) == S.SPARROW_EINVAL
    need = S.sparrow_residual_norm_workspace_size(3, 256)
    assert need >= 3 * 256 * 4
    assert backward(ws=None) == S.SPARROW_EWORKSPACE
    assert backward(ws=FAKE + 8) == S.SPARROW_EINVAL
    assert backward(n=need - 1) == S.SPARROW_EWORKSPACE
    for T, C in ((-1, 256), (1 << 31, 256), (3, 4), (3, 252), (3, 16392)):
        assert S.sparrow_residual_norm_workspace_size(T, C) == 0


def test_no_tokens_is_no_launch():
    assert forward(T=0) == S.SPARROW_OK
    assert backward(T=0) == S.SPARROW_OK


def test_wrappers_refuse_host_tensors_and_recorded_gradients():
    import torch
    z = torch.zeros(2, 64, dtype=torch.bfloat16)
    w = torch.ones(64, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="GPU"):
        S.residual_norm(z, z, w)
    with pytest.raises(RuntimeError, match="GPU"):
        S.residual_norm_bwd(z, z, z, z, w)
    for i in range(5):
        a = [z.clone(), z.clone(), w.clone(), w.clone(), z.clone()]
        a[i].requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            S.residual_norm(*a)
        with torch.no_grad(), pytest.raises(RuntimeError, match="GPU"):
            S.residual_norm(*a)
