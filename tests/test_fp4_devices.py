"""A launch goes to the current device, or to the one of the stream that is
passed: the 4-bit cache's calls refuse tensors of another."""
import types

import pytest
import torch

from paper_2607_13332_amd import ssn


class OnGpu:
    """What the wrappers look at of a tensor on GPU `index`."""

    def __init__(self, index, dtype, *shape):
        self.index, self.dtype, self.shape = index, dtype, torch.Size(shape)
        self.device, self.is_cuda = torch.device("cuda", index), True

    def get_device(self):
        return self.index

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self):
        return torch.empty(self.shape, device="meta").stride()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 32


class Library:
    """Counts the calls that reach the library."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a[-1])) or 0


def _calls(index):
    u8, i32, f32 = torch.uint8, torch.int32, torch.float32
    x, out = OnGpu(index, f32, 4, 2, 64), OnGpu(index, f32, 4, 2, 64)
    cache = [OnGpu(index, u8, 3, 2, 16, n) for n in (32, 2, 32, 2)]
    batch = OnGpu(index, i32, 1, 3), OnGpu(index, i32, 2), OnGpu(index, i32, 1)
    return [lambda **k: ssn.kv_append_fp4(x, x, *cache, *batch, **k),
            lambda **k: ssn.kv_read_fp4(*cache, *batch, 4, Kout=x, Vout=out, **k),
            lambda **k: ssn.paged_attention_fp4(x, *cache, *batch, 4, 4, out=out, **k)]


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(ssn, "lib", lambda: lib)
    monkeypatch.setattr(ssn, "_get_device", lambda: 0)
    monkeypatch.setattr(ssn, "_raw_current_stream", lambda device: 100 + device)
    return lib


@pytest.mark.parametrize("call", range(3))
def test_tensors_of_another_device(library, call):
    with pytest.raises(ValueError, match="the current device is 0"):
        _calls(1)[call]()
    assert not library.calls
    _calls(0)[call]()
    assert [s for _, s in library.calls] == [100]


@pytest.mark.parametrize("call", range(3))
def test_a_stream_of_another_device(library, call):
    stream = types.SimpleNamespace(cuda_stream=7, device_index=1)
    with pytest.raises(ValueError, match="stream is on GPU 1"):
        _calls(0)[call](stream=stream)
    assert not library.calls
    _calls(1)[call](stream=stream)            # theirs, whatever the current one
    _calls(0)[call](stream=types.SimpleNamespace(cuda_stream=9))
    assert [s for _, s in library.calls] == [7, 9]
    # the default stream has no handle of its own: it is the current device's
    with pytest.raises(ValueError, match="the current device is 0"):
        _calls(1)[call](stream=types.SimpleNamespace(cuda_stream=0, device_index=1))
    _calls(0)[call](stream=types.SimpleNamespace(cuda_stream=0, device_index=0))
    assert [s for _, s in library.calls] == [7, 9, 0]
