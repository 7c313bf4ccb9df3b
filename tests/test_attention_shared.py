"""sparrow_shared_prefix_decode_attn refuses bad host-visible arguments before any launch."""
import pytest

from paper_2606_08446_amd import sparrow as S

FAKE = 0x1000


def shape(**kw):
    d = dict(batch=4, num_q_heads=16, num_kv_heads=8, page_size=16, max_pages_per_seq=64,
             num_phys_pages=300) | kw
    return S.make_shape(**d)


def call(sh, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, bt=FAKE, lens=FAKE, n=2, cu=FAKE, pre=FAKE, scale=0.088, out=FAKE,
             dt=0, ws=FAKE, nb=1 << 40) | kw
    return S.sparrow_shared_prefix_decode_attn(sh, a["q"], a["k"], a["v"], a["bt"], a["lens"], a["n"],
                                               a["cu"], a["pre"], a["scale"], a["out"], a["dt"],
                                               a["ws"], a["nb"], None)


BAD_SHAPES = [(dict(head_dim=64), S.SPARROW_EUNSUPPORTED),
              (dict(num_q_heads=12, num_kv_heads=8), S.SPARROW_EINVAL),
              (dict(page_size=8), S.SPARROW_EUNSUPPORTED), (dict(page_size=48), S.SPARROW_EUNSUPPORTED),
              (dict(num_q_heads=136, num_kv_heads=8), S.SPARROW_EUNSUPPORTED),
              (dict(max_pages_per_seq=S.SPARROW_MAX_PAGES_PER_SEQ + 1), S.SPARROW_EUNSUPPORTED),
              (dict(batch=-1), S.SPARROW_EINVAL), (dict(num_phys_pages=0), S.SPARROW_EINVAL),
              (dict(batch=8192), S.SPARROW_EINVAL),            # 65536 (sequence, KV head) units
              (dict(batch=8193, num_kv_heads=1, num_q_heads=1), S.SPARROW_EUNSUPPORTED)]


@pytest.mark.parametrize("bad,status", BAD_SHAPES)
def test_bad_shapes(bad, status):
    bad = dict(bad)
    head_dim = bad.pop("head_dim", 128)
    sh = shape(**bad)
    sh.head_dim = head_dim
    assert call(sh) == status
    assert S.sparrow_shared_prefix_workspace_size(sh, 2) == 0


@pytest.mark.parametrize("name", ["q", "k", "v", "bt", "lens", "cu", "pre", "out"])
def test_pointers(name):
    assert call(shape(), **{name: None}) == S.SPARROW_EINVAL
    assert call(shape(), **{name: FAKE + 2}) == S.SPARROW_EINVAL


def test_groups_scale_dtype_and_workspace():
    sh = shape()
    assert call(sh, n=-1) == S.SPARROW_EINVAL
    assert call(sh, n=S.SPARROW_MAX_GROUPS + 1) == S.SPARROW_EUNSUPPORTED
    assert call(sh, scale=float("nan")) == S.SPARROW_EINVAL
    assert call(sh, scale=float("inf")) == S.SPARROW_EINVAL
    assert call(sh, dt=2) == S.SPARROW_EUNSUPPORTED
    need = S.sparrow_shared_prefix_workspace_size(sh, 2)
    assert need > 0
    assert call(sh, ws=None) == S.SPARROW_EWORKSPACE
    assert call(sh, nb=need - 1) == S.SPARROW_EWORKSPACE
    assert call(sh, ws=FAKE + 8) == S.SPARROW_EINVAL
    assert S.sparrow_shared_prefix_workspace_size(sh, -1) == 0
    assert S.sparrow_shared_prefix_workspace_size(sh, S.SPARROW_MAX_GROUPS + 1) == 0
    assert S.sparrow_shared_prefix_workspace_size(sh, 0) > 0


def test_an_empty_batch_is_no_launch():
    assert call(shape(batch=0)) == S.SPARROW_OK


def test_wrapper_refuses_host_tensors():
    import torch
    z = torch.zeros(2, 4, 128, dtype=torch.bfloat16)
    c = torch.zeros(8, 2, 16, 128, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(RuntimeError, match="GPU"):
        S.shared_prefix_decode_attn(z, c, c, torch.zeros(2, 4, dtype=torch.int32), i, i, i[:1])
