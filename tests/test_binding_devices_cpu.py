"""A model's weights and the tensors of a call have to be on one device: kernels would read the other device's memory (stand-ins for tensors;
no GPU needed)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2601_15013_amd import binding

LAUNCHED = "launched"


class Tensor:
    """What the binding asks of a CUDA tensor."""
    is_cuda = True

    def __init__(self, shape, dtype, index):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", index)

    def dim(self): return len(self.shape)
    def numel(self): return self.shape.numel()
    def is_contiguous(self): return True
    def get_device(self): return self.device.index
    def data_ptr(self): return 0x1000


@pytest.fixture
def calls(monkeypatch):
    def launch(*a):
        raise RuntimeError(LAUNCHED)

    monkeypatch.setattr(binding, "_launch", launch)
    monkeypatch.setattr(binding, "_new_all", lambda outputs, device, stream: [Tensor(shape, dtype, device.index) for shape, dtype in outputs])
    monkeypatch.setattr(binding, "_new", lambda shape, dtype, device, stream: Tensor(shape, dtype, device.index))

    def model(index):
        m = binding.Model(0, SimpleNamespace(d=64), index)
        return m

    def extend(index, at):
        i32 = lambda n: Tensor((n,), torch.int32, at)
        cache = SimpleNamespace(device=torch.device("cuda", at), ref=None)
        binding.radix_extend_forward(model(index), cache, i32(5), i32(2), 5, Tensor((99,), torch.uint8, at))

    def score(index, at):
        binding.radix_score_tokens(model(index), Tensor((5, 64), torch.float32, at), None, None, Tensor((99,), torch.uint8, at), top_k=1)

    return extend, score


@pytest.mark.parametrize("call", [0, 1])
def test_a_model_of_another_device_is_refused(calls, call):
    for index, at in ((0, 1), (1, 0)):
        with pytest.raises(ValueError, match=f"cuda:{index}"):
            calls[call](index, at)
    for index in (0, 1):
        with pytest.raises(RuntimeError, match=LAUNCHED):
            calls[call](index, index)
