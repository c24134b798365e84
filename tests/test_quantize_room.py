"""The rows of the transposed 8-bit form are written in whole runs of 16 bytes: a tensor whose memory ends before is refused.
(Host tensors that say they are on a GPU: the rule looks at properties only.)"""
import pytest
import torch

import paper_2509_25401_amd as pkg
from paper_2509_25401_amd import block


class OnGpu:
    def __init__(self, t):
        self.t = t

    is_cuda = True
    get_device = lambda self: 0
    __getattr__ = lambda self, name: getattr(self.t, name)


class Taken(Exception):
    pass


@pytest.fixture
def quantize(monkeypatch):
    lib = block._library()

    class Library:
        def __getattr__(self, name):
            return getattr(lib, name)

        def sparse_fp8_quantize(self, *args):
            raise Taken(*args)

    monkeypatch.setattr(block, "_lib", Library())
    monkeypatch.setattr(block, "_stream_ptr", lambda stream: None)

    def call(R, C, qt):
        scales = torch.zeros(C, -(-R // 128), dtype=torch.uint8)
        pkg.sparse_fp8_quantize(OnGpu(torch.zeros(R, C, dtype=torch.bfloat16)), None, None, OnGpu(qt), OnGpu(scales))

    return call


def _bytes(n, offset, shape, strides):
    return torch.zeros(n, dtype=torch.uint8).view(torch.float8_e4m3fn).as_strided(shape, strides, offset)


@pytest.mark.parametrize("R,C,qt", [
    (5, 1, torch.zeros(1, 5, dtype=torch.float8_e4m3fn)),                # one row: five bytes, sixteen would be written
    (33, 1, _bytes(64, 20, (1, 33), (64, 1))),
    (40, 3, _bytes(2 * 48 + 40, 0, (3, 40), (48, 1))),                   # the last row ends with its last value
    (1, 4, _bytes(49, 0, (4, 1), (16, 1))),
])
def test_memory_that_ends_early(quantize, R, C, qt):
    with pytest.raises(ValueError, match="memory of qt"):
        quantize(R, C, qt)


@pytest.mark.parametrize("R,C,qt", [
    (5, 1, torch.zeros(1, 16, dtype=torch.float8_e4m3fn)[:, :5]),
    (16, 1, torch.zeros(1, 16, dtype=torch.float8_e4m3fn)),
    (40, 3, torch.zeros(3, 48, dtype=torch.float8_e4m3fn)[:, :40]),
    (48, 3, torch.zeros(3, 48, dtype=torch.float8_e4m3fn)),
    (1, 4, _bytes(64, 0, (4, 1), (16, 1))),
])
def test_memory_that_suffices(quantize, R, C, qt):
    with pytest.raises(Taken) as call:
        quantize(R, C, qt)
    assert call.value.args[3] == qt.data_ptr() and call.value.args[5] == (qt.stride(0) if C > 1 else 16)
