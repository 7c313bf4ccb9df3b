"""sparrow_sample refuses bad host-visible arguments before any launch."""
import pytest

from paper_2606_08446_amd import sparrow as S

FAKE = 0x1000
BAD = [(dict(T=-1), S.SPARROW_EINVAL), (dict(T=1 << 31), S.SPARROW_EINVAL),
       (dict(V=0, stride=0), S.SPARROW_EINVAL), (dict(V=-5), S.SPARROW_EINVAL),
       (dict(V=S.SPARROW_SAMPLE_MAX_VOCAB + 1, stride=1 << 20), S.SPARROW_EUNSUPPORTED),
       (dict(stride=999), S.SPARROW_EINVAL), (dict(stride=-1000), S.SPARROW_EINVAL),
       (dict(dt=2), S.SPARROW_EUNSUPPORTED), (dict(dt=-1), S.SPARROW_EUNSUPPORTED)]


def call(**kw):
    a = dict(T=3, V=1000, dt=0, z=FAKE, stride=1003, t=FAKE, k=FAKE, p=FAKE, q=FAKE, u=FAKE, tok=FAKE,
             lp=FAKE, ws=FAKE, n=1 << 40) | kw
    return S.sparrow_sample(a["T"], a["V"], a["dt"], a["z"], a["stride"], a["t"], a["k"], a["p"],
                            a["q"], a["u"], a["tok"], a["lp"], a["ws"], a["n"], None)


@pytest.mark.parametrize("bad,status", BAD)
def test_bad_sizes_are_refused(bad, status):
    assert call(**bad) == status


@pytest.mark.parametrize("name", ["z", "u", "tok"])
def test_null_pointers(name):
    assert call(**{name: None}) == S.SPARROW_EINVAL


@pytest.mark.parametrize("name", ["z", "t", "k", "p", "q", "u", "tok", "lp"])
def test_alignment(name):
    assert call(**{name: FAKE + 2}) == S.SPARROW_EINVAL
    assert call(dt=1, z=FAKE + 1) == S.SPARROW_EINVAL


def test_workspace():
    for dt in (0, 1):
        need = S.sparrow_sample_workspace_size(3, 1000, dt)
        assert need > 0
        assert call(dt=dt, ws=None) == S.SPARROW_EWORKSPACE
        assert call(dt=dt, ws=FAKE + 8) == S.SPARROW_EINVAL
        assert call(dt=dt, n=need - 1) == S.SPARROW_EWORKSPACE
    for bad in ((-1, 1000, 0), (1 << 31, 1000, 0), (3, 0, 0),
                (3, S.SPARROW_SAMPLE_MAX_VOCAB + 1, 0), (3, 1000, 2)):
        assert S.sparrow_sample_workspace_size(*bad) == 0


def test_no_rows_is_no_launch():
    assert call(T=0) == S.SPARROW_OK


def test_wrapper_refuses_host_tensors():
    import torch
    with pytest.raises(RuntimeError, match="GPU"):
        S.sample(torch.zeros(2, 10), torch.zeros(2))
