"""The gradient of the norms around a block where a workgroup has several rows: the loop behind the first row, its
rows in turn, and the weights' sums over all of them, in every variant.  Against the formulas in 64 bits."""
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log
from test_gpu_residual_norm import check_backward, grad, make

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


# Rows a workgroup: odd and even numbers of them side by side, where the tokens are no multiple of the 256 to 2048
# workgroups.  One vector a thread; two, with sums in registers; sums in LDS above 8192 channels.  A channel's
# sum is a chain of at most 10 rows, 64 workgroups and 32 parts: the 150 steps that the bound has.
SHAPES = [(4099, 256), (9001, 1016), (4500, 1024), (2600, 2056), (1300, 4096), (1021, 5120), (600, 8192),
          (700, 8200), (515, 16384)]


@pytest.mark.parametrize("T,C", SHAPES)
@pytest.mark.parametrize("post,gate", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32])
def test_several_rows_a_workgroup(T, C, post, gate, stream):
    log(f"case residual_norm rows T={T} C={C} post={post} gate={gate} {stream}")
    d, dy, dh = make(T, C, T + C, post, gate, stream)
    if not post and not gate:
        d["x"] = d["x"].contiguous()
    check_backward(d, dy, dh, grad(dy, dh, d))
    if post and gate:
        check_backward(d, dy, None, grad(dy, None, d))


# Results of 224 MB and more, which are stored past the caches: 19 rows a workgroup (chains of 19, 16 and 32) of
# 4096 channels, 16 (16, 8 and 32) of 10000 with the sums in LDS.
@pytest.mark.parametrize("T,C", [(9601, 4096), (4001, 10000)])
def test_results_past_the_caches(T, C):
    log(f"case residual_norm past the caches T={T} C={C}")
    assert T * C * 6 >= 224 << 20
    d, dy, dh = make(T, C, 7)
    check_backward(d, dy, dh, grad(dy, dh, d))
