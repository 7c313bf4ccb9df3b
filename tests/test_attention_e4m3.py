"""The attention calls over an e4m3 cache refuse bad host-visible arguments before any launch."""
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from test_abi import BAD_SHAPES, FAKE, good_shape


def call(sparse, shape=None, **kw):
    a = dict(q=FAKE, kc=FAKE, vc=FAKE, e=FAKE, bt=FAKE, lens=FAKE, k=FAKE, idx=FAKE, k_max=8,
             out=FAKE, dt=0, ws=FAKE, n=1 << 40) | kw
    shape = shape or good_shape()
    if sparse:
        return S.sparrow_sparse_decode_attn_e4m3(
            shape, a["q"], a["kc"], a["vc"], a["e"], a["bt"], a["lens"], a["k"], a["idx"],
            a["k_max"], 0.088, a["out"], a["dt"], a["ws"], a["n"], None)
    return S.sparrow_dense_decode_attn_e4m3(shape, a["q"], a["kc"], a["vc"], a["e"], a["bt"],
                                            a["lens"], 0.088, a["out"], a["dt"], a["ws"], a["n"],
                                            None)


@pytest.mark.parametrize("sparse", [False, True])
@pytest.mark.parametrize("bad,status", BAD_SHAPES)
def test_bad_shapes(sparse, bad, status):
    bad = dict(bad)
    head_dim = bad.pop("head_dim", 128)
    shape = good_shape(**bad)
    shape.head_dim = head_dim
    assert call(sparse, shape) == status


@pytest.mark.parametrize("name", ["q", "kc", "vc", "e", "bt", "lens", "k", "idx", "out"])
def test_pointers(name):
    for sparse in ((True,) if name in ("k", "idx") else (False, True)):
        assert call(sparse, **{name: None}) == S.SPARROW_EINVAL
        assert call(sparse, **{name: FAKE + 2}) == S.SPARROW_EINVAL
        if name in ("q", "kc", "vc", "e", "out"):
            assert call(sparse, **{name: FAKE + 4}) == S.SPARROW_EINVAL


@pytest.mark.parametrize("sparse", [False, True])
def test_other_refusals(sparse):
    need = S.sparrow_workspace_size(good_shape(), 8, S.SPARROW_OP_DENSE_ATTN)
    assert call(sparse, dt=2) == S.SPARROW_EUNSUPPORTED
    assert call(sparse, ws=None) == S.SPARROW_EWORKSPACE
    assert call(sparse, n=need - 1) == S.SPARROW_EWORKSPACE
    assert call(sparse, ws=FAKE + 4) == S.SPARROW_EINVAL
    assert call(sparse, good_shape(batch=0), ws=None) == S.SPARROW_OK
    assert call(sparse, good_shape(batch=S.SPARROW_MAX_BATCH + 1)) == S.SPARROW_EUNSUPPORTED
    # 16-token parts of the cache are numbered in 32 bits
    assert call(sparse, good_shape(num_phys_pages=1 << 28, batch=0)) == S.SPARROW_OK
    assert call(sparse, good_shape(num_phys_pages=1 << 28)) == S.SPARROW_EUNSUPPORTED
    assert call(sparse, good_shape(num_phys_pages=1 << 25, page_size=128)) == S.SPARROW_EUNSUPPORTED
    if sparse:
        assert call(True, k_max=0) == S.SPARROW_EINVAL
        assert call(True, k_max=S.SPARROW_MAX_PAGES_PER_SEQ + 1) == S.SPARROW_EINVAL


def test_wrappers_refuse_host_tensors():
    k, v, e = S.new_cache_e4m3(3, 2, 16, "cpu")
    q = torch.zeros(1, 4, 128, dtype=torch.bfloat16)
    bt, lens = torch.zeros(1, 2, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    with pytest.raises(RuntimeError):
        S.dense_decode_attn_e4m3(q, k, v, e, bt, lens)
    with pytest.raises(RuntimeError):
        S.sparse_decode_attn_e4m3(q, k, v, e, bt, lens, lens, torch.zeros(1, 2, 2, dtype=torch.int32))
    with pytest.raises(ValueError):
        S.sparse_decode_attn_e4m3(q, k, v, e, bt, lens, lens, None)
