"""What the binding of the language-model operators refuses before a launch, on the CPU: stand-ins have the attributes of CUDA tensors, and the
library's calls are recorded instead of made."""
import math
from types import SimpleNamespace

import pytest
import torch

from paper_2007_06919_gb300 import aqd


class Tensor:
    """A tensor of one storage on device `index` (None: the host)."""
    def __init__(self, shape, dtype, index=0, strides=None):
        self.shape, self.dtype, self.index = torch.Size(shape), dtype, index
        self.is_cuda = index is not None
        self.device = torch.device("cpu") if index is None else torch.device("cuda", index)
        contiguous = [math.prod(shape[i + 1:]) for i in range(len(shape))]
        self.strides = contiguous if strides is None else strides
        self.contiguous = list(self.strides) == contiguous
        self.nbytes = math.prod(shape) * dtype.itemsize

    def stride(self):
        return tuple(self.strides)

    def get_device(self):
        return -1 if self.index is None else self.index

    def numel(self):
        return math.prod(self.shape)

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 0x7000_0000_0000

    def __getitem__(self, _):
        return self


@pytest.fixture
def made(monkeypatch):
    """The names of the calls that reached the library; the current device is 0."""
    names = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                names.append(name)
                return 1 << 20 if name.endswith("_bytes") else 0
            return call

    monkeypatch.setattr(aqd, "_calls", Library)
    monkeypatch.setattr(aqd, "_raw_device", lambda: 0)
    monkeypatch.setattr(aqd, "_stream", lambda s=None: 0)
    monkeypatch.setattr(aqd, "_new", lambda shape, dtype, device, stream: Tensor((shape,) if isinstance(shape, int) else shape, dtype, device.index))
    return names


def layer(index=0):
    return SimpleNamespace(n=64, k=128, index=index, device=torch.device("cuda", index), desc=b"", scales=None)


def codes(index=0):
    return Tensor((4, 128), torch.int8, index), Tensor((4,), torch.float32, index)


@pytest.mark.parametrize("space", [Tensor((1 << 20,), torch.uint8, None), Tensor((1 << 20,), torch.uint8, 1),
                                   Tensor((1 << 10, 1 << 10), torch.uint8, 0, (1 << 11, 1)), Tensor((1 << 20,), torch.uint8, 0, (2,))])
def test_a_workspace_that_the_kernels_cannot_write(made, space):
    with pytest.raises(ValueError, match="workspace"):
        aqd.linear_int8(*codes(), layer(), workspace=space)
    assert made == []


def test_a_workspace_of_any_type(made):
    for space in (Tensor((1 << 20,), torch.uint8), Tensor((64, 1 << 10), torch.float32), None):
        aqd.linear_int8(*codes(), layer(), workspace=space)
    assert made == ["aqd_linear_int8"] * 3


def matrix(index=0, dtype=torch.float32, cols=128):
    return Tensor((4, cols), dtype, index)


def vector(n, index=0, dtype=torch.float32):
    return Tensor((n,), dtype, index)


CALLS = {
    "quant_rows": lambda d, s: aqd.quant_rows(matrix(d), stream=s),
    "rms_norm_quant": lambda d, s: aqd.rms_norm_quant(matrix(d), vector(128, d), residual=matrix(d), stream=s),
    "gated_act_quant": lambda d, s: aqd.gated_act_quant(matrix(d), matrix(d), stream=s),
    "LinearWeights": lambda d, s: aqd.LinearWeights(matrix(d, torch.int8), vector(4, d), stream=s),
    "linear_int8": lambda d, s: aqd.linear_int8(*codes(d), layer(d), stream=s),
    "distill_topk": lambda d, s: aqd.distill_topk(matrix(d), matrix(d, torch.int64, 8), matrix(d, cols=8), grad=True, stream=s),
    "distill_topk_backward": lambda d, s: aqd.distill_topk_backward(matrix(d), matrix(d, torch.int64, 8), matrix(d, cols=8), vector(4, d), stream=s),
}


@pytest.mark.parametrize("call", list(CALLS))
def test_tensors_and_streams_of_another_device_than_the_current_one(made, call):
    """The kernels would run on the current device whatever the addresses are of."""
    here, there = (SimpleNamespace(device=torch.device("cuda", i), cuda_stream=5) for i in (0, 1))
    for d, s in ((1, None), (1, there), (0, there), (1, here)):
        with pytest.raises(ValueError, match="device"):
            CALLS[call](d, s)
    assert [n for n in made if not n.endswith("_bytes")] == []
    CALLS[call](0, None)
    CALLS[call](0, here)
    assert len([n for n in made if not n.endswith("_bytes")]) == 2
