"""The e4m3 cache on the host: the test helpers' own format against torch's float8 cast, and the
entry points' refusals before any launch."""
import numpy as np
import pytest
import torch

import e4m3
from paper_2606_08446_amd import sparrow as S

from test_abi import BAD_SHAPES, FAKE, good_shape


def test_the_grid_is_torchs_e4m3():
    x = np.concatenate([np.linspace(-448, 448, 20001), np.ldexp(np.linspace(-2, 2, 2001), -9)])
    x = np.concatenate([x, np.zeros(-len(x) % 127)]).astype(np.float32).reshape(-1, 127)
    x = np.concatenate([x, np.full((len(x), 1), 448.0, np.float32)], 1)    # every row's e is 0
    y, e = e4m3.quantise(x)
    assert (e == 0).all()
    want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(y, want)


def test_exponents_at_their_edges():
    for top, e in ((448.0, 0), (449.0, 1), (1.75, -8), (1.76, -7), (0.0, -117), (2.0 ** -125, -117),
                   (2.0 ** 127, 119), (1.75 * 2.0 ** 127, 119), (1.99 * 2.0 ** 127, 119)):
        x = np.zeros(128)
        x[5] = -top
        assert e4m3.quantise(x)[1] == e, top


def append(shape=None, **kw):
    a = dict(k=FAKE, ks=1024, v=FAKE, vs=1024, cu=FAKE, T=10, kc=FAKE, vc=FAKE, e=FAKE, bt=FAKE,
             lens=FAKE, meta=FAKE) | kw
    return S.sparrow_append_kv_e4m3(shape or good_shape(), a["k"], a["ks"], a["v"], a["vs"],
                                    a["cu"], a["T"], a["kc"], a["vc"], a["e"], a["bt"], a["lens"],
                                    a["meta"], None)


def read(shape=None, **kw):
    a = dict(kc=FAKE, vc=FAKE, e=FAKE, bt=FAKE, lens=FAKE, cu=FAKE, T=10, k=FAKE, v=FAKE) | kw
    return S.sparrow_read_kv_e4m3(shape or good_shape(), a["kc"], a["vc"], a["e"], a["bt"],
                                  a["lens"], a["cu"], a["T"], a["k"], a["v"], None)


@pytest.mark.parametrize("bad,status", BAD_SHAPES)
def test_bad_shapes(bad, status):
    bad = dict(bad)
    head_dim = bad.pop("head_dim", 128)
    shape = good_shape(**bad)
    shape.head_dim = head_dim
    assert append(shape) == status and read(shape) == status


@pytest.mark.parametrize("name", ["k", "v", "kc", "vc", "e", "bt", "lens", "meta"])
def test_append_pointers(name):
    assert append(**{name: None}) == S.SPARROW_EINVAL
    assert append(**{name: FAKE + 2}) == S.SPARROW_EINVAL
    if name not in ("bt", "lens"):
        assert append(**{name: FAKE + 4}) == S.SPARROW_EINVAL
    assert append(cu=FAKE + 2) == S.SPARROW_EINVAL


@pytest.mark.parametrize("name", ["k", "v", "kc", "vc", "e", "bt", "lens"])
def test_read_pointers(name):
    assert read(**{name: None}) == S.SPARROW_EINVAL
    assert read(**{name: FAKE + 2}) == S.SPARROW_EINVAL
    assert read(cu=FAKE + 2) == S.SPARROW_EINVAL


def test_rows():
    for f in (append, read):
        assert f(T=-1) == S.SPARROW_EINVAL
        assert f(T=(1 << 27) + 1) == S.SPARROW_EINVAL
        assert f(cu=None, T=5) == S.SPARROW_EINVAL        # one row per sequence: 4 of them
        assert f(T=0) == S.SPARROW_OK
        assert f(good_shape(batch=0), T=0) == S.SPARROW_OK
        assert f(good_shape(batch=(1 << 20) + 1)) == S.SPARROW_EINVAL
        assert f(good_shape(num_q_heads=65536, num_kv_heads=65536)) == S.SPARROW_EINVAL
    assert append(ks=1016) == S.SPARROW_EINVAL
    assert append(vs=1028) == S.SPARROW_EINVAL


def test_wrappers_refuse_host_tensors():
    k, v, e = S.new_cache_e4m3(3, 2, 16, "cpu")
    bt, lens = torch.zeros(1, 2, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    rows = torch.zeros(1, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError):
        S.append_kv_e4m3(rows, rows, k, v, e, bt, lens, S.new_meta(3, 2, "cpu"))
    with pytest.raises(RuntimeError):
        S.read_kv_e4m3(k, v, e, bt, lens, None, 1)
