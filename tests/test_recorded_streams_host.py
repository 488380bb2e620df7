"""On which streams an object records the tensors it keeps, on stand-ins."""
import pytest
import torch

from paper_2502_03805_b200 import cache as cache_module


class Stream:
    def __init__(self, cuda_stream, stream_id):
        self.cuda_stream, self.stream_id = cuda_stream, stream_id


class Tensor:
    def __init__(self):
        self.on = []

    def record_stream(self, s):
        self.on.append(s)


class Owner(cache_module._Owner):
    def __init__(self):
        self._index, self.device, self._seen, self.tensor = 0, torch.device("cuda", 0), set(), Tensor()

    def _kept(self):
        return (None, self.tensor)


@pytest.fixture
def current(monkeypatch):
    s = Stream(0x1000, 35)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: s)
    monkeypatch.setattr(cache_module, "_raw_stream", lambda index: s.cuda_stream)
    default = Stream(0, 0)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: default)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda at, device=None: Stream(at, at))
    return s, default


def test_torch_streams_are_recorded_once(current):
    s, default = current
    o, other = Owner(), Stream(0x2000, 67)
    assert [o._where(x) for x in (None, None, other, s, other, 0, default)] == [0x1000, 0x1000, 0x2000, 0x1000, 0x2000, 0, 0]
    assert o.tensor.on == [s, other, default]


def test_streams_that_torch_did_not_make_are_not(current):
    """Their owner may have destroyed them by the time the tensor goes."""
    o = Owner()
    assert o._where(0x3000) == 0x3000 and o._where(Stream(0x4000, 0x4000)) == 0x4000
    current[0].stream_id = current[0].cuda_stream            # the current stream, too
    assert o._where(None) == 0x1000
    assert o.tensor.on == []
