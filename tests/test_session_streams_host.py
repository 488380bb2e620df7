"""In which order the streams of a session and of a cache wait for each other, on stand-ins that write down what happens."""
import contextlib

import pytest
import torch

from paper_2502_03805_b200 import ChunkedPrefillCompressor, CompressionSession


class Stream:
    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append((self.name, "waits for", other.name))


class Cache:
    nseq, Hkv, device = 1, 2, "cpu"

    def __init__(self, log):
        self.log = log

    def _allocating(self, stream):
        return contextlib.nullcontext()

    def new_lengths(self):
        return torch.zeros(1, 2, dtype=torch.int32)

    def store(self, K, V, start, lens_out=None, *, idx=None, offsets=None, counts=None, stream=None):
        self.log.append(("store on", stream))
        return torch.zeros(1, 2, dtype=torch.int32) if lens_out is None else lens_out


@pytest.fixture(params=["default", "side"])
def streams(request, monkeypatch):
    log = []
    made = {n: Stream(n, log) for n in ("default", "side")}
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: made["default"])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: made[request.param])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return request.param, log


def test_compact_into_waits_for_the_current_stream_and_is_waited_for(streams):
    current, log = streams
    s = object.__new__(CompressionSession)
    s.handle, s.device, s.btot = None, "cpu", 4
    s.idx, s.offsets = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, 3, dtype=torch.int32)
    K = torch.zeros(1, 2, 4, 64)
    lens = s.compact_into(Cache(log), K, K, torch.zeros(1, 2, dtype=torch.int32))
    assert lens.shape == (1, 2) and lens.dtype == torch.int32
    inside = [("store on", 0)]
    assert log == (inside if current == "default" else
                   [("default", "waits for", "side")] + inside + [("side", "waits for", "default")])
    log.clear()
    s.compact_into(Cache(log), K, K, lens, lens, stream=77)      # a stream of the caller's: its own order
    assert log == [("store on", 77)]


@pytest.mark.parametrize("mode", ["uniform", "adaptive"])
def test_to_cache_waits_for_the_stream_of_the_steps(streams, mode):
    current, log = streams
    ch = ChunkedPrefillCompressor(Hq=2, Hkv=2, dh=64, dm=64, w=8, pool_k=3, dtype="f32", budget_mode=mode)
    ch.device = torch.device("cpu")
    K = torch.zeros(2, 3, 64)
    ch.K, ch.V = (K, K) if mode == "uniform" else (list(K), list(K))
    ch.to_cache(Cache(log))
    assert log == ([] if current == "default" else [("side", "waits for", "default")]) + [("store on", None)]
    log.clear()
    ch.to_cache(Cache(log), stream=77)
    assert log == [("store on", 77)]


def test_while_the_current_stream_is_captured(streams, monkeypatch):
    """The default stream cannot be captured: neither waits for the other, and what would run on it is refused."""
    current, log = streams
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    s = object.__new__(CompressionSession)
    s.handle, s.device, s.btot = None, "cpu", 4
    s.idx, s.offsets = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, 3, dtype=torch.int32)
    ch = ChunkedPrefillCompressor(Hq=2, Hkv=2, dh=64, dm=64, w=8, pool_k=3, dtype="f32")
    ch.device = torch.device("cpu")
    K = ch.K = ch.V = torch.zeros(2, 3, 64)
    ch.to_cache(Cache(log))
    assert log == [("store on", None)]
    log.clear()
    start = torch.zeros(1, 2, dtype=torch.int32)
    if current == "side":
        with pytest.raises(ValueError):
            s.compact_into(Cache(log), K, K, start)
        assert log == []
    s.compact_into(Cache(log), K, K, start, stream=77)
    assert log == [("store on", 77)]
