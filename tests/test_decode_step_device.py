"""SparseDecodeStep launches with its tensors' device as the current one (on the host: the library's
calls and the devices are stand-ins)."""
import types

import pytest
import torch

from paper_2606_08446_amd import sparrow as S


class Tensor:
    """What the wrappers ask of a tensor on a device of this machine or of none."""
    is_cuda = True

    def __init__(self, dtype, *shape):
        self.dtype, self.shape, self.device = dtype, torch.Size(shape), torch.device("cuda", 1)

    def dim(self):
        return len(self.shape)

    def stride(self):
        return tuple(self.shape[i + 1:].numel() for i in range(len(self.shape)))

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def numel(self):
        return self.shape.numel()


def make(monkeypatch, e4m3, at):
    """A step on device 1 with device ``at[0]`` current, and the list that its launches go to."""
    made = []
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: Tensor(
        dtype, *(shape if hasattr(shape, "__iter__") else (shape,))))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: at[0])

    class device:
        def __init__(self, to):
            self.to = torch.device(to).index

        def __enter__(self):
            self.old, at[0] = at[0], self.to

        def __exit__(self, *exc):
            at[0] = self.old
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: types.SimpleNamespace(cuda_stream=0))
    for name in ("page_meta_update", "append_kv", "append_kv_e4m3", "page_score_topk",
                 "append_score_topk", "sparse_decode_attn", "sparse_decode_attn_e4m3", "decode_step"):
        def launch(*args, name=name):
            made.append((name, at[0]))
            return S.SPARROW_OK
        monkeypatch.setattr(S, "sparrow_" + name, launch)
    i32, bf, cache = torch.int32, torch.bfloat16, (6, 2, 16, 128)
    k, v = (Tensor(torch.float8_e4m3fn if e4m3 else bf, *cache) for _ in range(2))
    step = S.SparseDecodeStep(
        Tensor(bf, 3, 8, 128), k, v, Tensor(i32, 3, 2), Tensor(i32, 3), Tensor(bf, 6, 2, 2, 128),
        Tensor(i32, 1), Tensor(i32, 1), 10, 2048, 2, exps=Tensor(torch.uint8, 6, 2, 4, 2, 4) if e4m3 else None)
    return step, made


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("current", [0, 1])
def test_launches_are_on_the_tensors_device(monkeypatch, e4m3, current):
    at = [current]
    step, made = make(monkeypatch, e4m3, at)
    new = [Tensor(torch.bfloat16, 3, 2, 128) for _ in range(2)]
    step.append(*new, 0)
    step.score_topk(0)
    step.attend(0)
    step.append_score_topk(*new, 0)
    step.decode_step(*new, 0)
    step.decode_step(None, None, 0)
    step.run()
    if not e4m3:
        step.meta_update(None, 0)
    assert len(made) >= 9 and all(d == 1 for _, d in made), made
    assert at == [current]
    with pytest.raises(ValueError):
        step.append(new[0], Tensor(torch.float32, 3, 2, 128), 0)
    assert at == [current]
