"""sparrow_qk_norm_rope and its gradient refuse bad host-visible arguments before any launch."""
import pytest

from paper_2606_08446_amd import sparrow as S

FAKE = 0x1000
BAD = [(dict(T=-1), S.SPARROW_EINVAL), (dict(T=1 << 31), S.SPARROW_EINVAL),
       (dict(hq=0), S.SPARROW_EINVAL), (dict(hk=0), S.SPARROW_EINVAL),
       (dict(hq=1025, qs=1025 * 128), S.SPARROW_EINVAL),
       (dict(hk=1025, ks=1025 * 128), S.SPARROW_EINVAL),
       (dict(D=64), S.SPARROW_EUNSUPPORTED),
       (dict(qs=4 * 128 - 8), S.SPARROW_EINVAL), (dict(qs=4 * 128 + 4), S.SPARROW_EINVAL),
       (dict(ks=2 * 128 - 8), S.SPARROW_EINVAL), (dict(ks=-2048), S.SPARROW_EINVAL),
       (dict(eps=-1e-6), S.SPARROW_EINVAL), (dict(eps=float("nan")), S.SPARROW_EINVAL),
       (dict(eps=float("inf")), S.SPARROW_EINVAL)]
POINTERS = ["q", "k", "wq", "wk", "f", "pos"]


def forward(**kw):
    a = dict(T=3, hq=4, hk=2, D=128, q=FAKE, qs=1024, k=FAKE, ks=1024, wq=FAKE, wk=FAKE, f=FAKE,
             pos=FAKE, eps=1e-6, qo=FAKE, ko=FAKE) | kw
    return S.sparrow_qk_norm_rope(a["T"], a["hq"], a["hk"], a["D"], a["q"], a["qs"], a["k"],
                                  a["ks"], a["wq"], a["wk"], a["f"], a["pos"], a["eps"], a["qo"],
                                  a["ko"], None)


def backward(**kw):
    a = dict(T=3, hq=4, hk=2, D=128, dqo=FAKE, dko=FAKE, q=FAKE, qs=1024, k=FAKE, ks=1024, wq=FAKE,
             wk=FAKE, f=FAKE, pos=FAKE, eps=1e-6, dq=FAKE, dqs=512, dk=FAKE, dks=256, dwq=FAKE,
             dwk=FAKE, ws=FAKE, n=S.SPARROW_ROPE_WORKSPACE_BYTES) | kw
    return S.sparrow_qk_norm_rope_bwd(
        a["T"], a["hq"], a["hk"], a["D"], a["dqo"], a["dko"], a["q"], a["qs"], a["k"], a["ks"],
        a["wq"], a["wk"], a["f"], a["pos"], a["eps"], a["dq"], a["dqs"], a["dk"], a["dks"],
        a["dwq"], a["dwk"], a["ws"], a["n"], None)


@pytest.mark.parametrize("bad,status", BAD)
def test_bad_sizes_are_refused(bad, status):
    assert forward(**bad) == status
    assert backward(**bad) == status


@pytest.mark.parametrize("name", POINTERS + ["qo", "ko"])
def test_forward_pointers(name):
    assert forward(**{name: None}) == S.SPARROW_EINVAL
    assert forward(**{name: FAKE + 2}) == S.SPARROW_EINVAL
    if name != "pos":
        assert forward(**{name: FAKE + 4}) == S.SPARROW_EINVAL


@pytest.mark.parametrize("name", POINTERS + ["dqo", "dko", "dq", "dk", "dwq", "dwk"])
def test_backward_pointers(name):
    assert backward(**{name: None}) == S.SPARROW_EINVAL
    assert backward(**{name: FAKE + 2}) == S.SPARROW_EINVAL


def test_backward_strides_and_workspace():
    assert backward(dqs=504) == S.SPARROW_EINVAL
    assert backward(dks=260) == S.SPARROW_EINVAL
    assert backward(ws=None) == S.SPARROW_EWORKSPACE
    assert backward(ws=FAKE + 8) == S.SPARROW_EINVAL
    assert backward(n=S.SPARROW_ROPE_WORKSPACE_BYTES - 1) == S.SPARROW_EWORKSPACE


def test_no_tokens_is_no_launch():
    assert forward(T=0) == S.SPARROW_OK


def test_wrappers_refuse_host_tensors():
    import torch
    z = torch.zeros(2, 4, 128, dtype=torch.bfloat16)
    w = torch.ones(128, dtype=torch.bfloat16)
    f = torch.ones(64, dtype=torch.float64)
    pos = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(RuntimeError):
        S.qk_norm_rope(z, z, w, w, f, pos)
    with pytest.raises(RuntimeError):
        S.qk_norm_rope_bwd(z, z, z, z, w, w, f, pos)
