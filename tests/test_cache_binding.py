"""What the cache's Python entry points do on the host before a call: where its memory comes from.  No GPU needed: torch's device calls are
replaced by ones that note what they are asked for."""

import contextlib

import pytest
import torch

from paper_2511_23113_amd import binding as B

POOL = 0x5000          # a stream of torch's pool, which ExternalStream(0) gives out: a handle of 0 counts as none


class Stream:
    def __init__(self, raw, device=torch.device("cuda", 0)):
        self.cuda_stream, self.device = raw, device


class Noted:
    """A tensor that knows the stream that it was allocated on."""

    def __init__(self, raw):
        self.raw, self.recorded = raw, []

    def record_stream(self, stream):
        self.recorded.append(stream.cuda_stream)


@pytest.fixture
def cache(monkeypatch):
    B._torch_module()
    entered = []

    @contextlib.contextmanager
    def on(stream):
        entered.append(stream.cuda_stream)
        yield
        entered.pop()
    now = Stream(0x7000)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: now.cuda_stream, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream(0))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw, device=None: Stream(raw or POOL))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: Noted(entered[-1] if entered else now.cuda_stream))
    c = object.__new__(B.KVCache)
    c.device, c._index = torch.device("cuda", 0), 0
    return c


@pytest.mark.parametrize("stream, raw, recorded", [(None, 0x7000, []), (Stream(0x7000), 0x7000, []), (Stream(0x9000), 0x9000, [0x7000]), (0x9000, 0x9000, [0x7000]),
                                                   (Stream(0), 0, [0x7000]), (0, 0, [0x7000])])
def test_a_calls_memory_comes_from_the_stream_that_its_kernels_run_on(cache, stream, raw, recorded):
    got, elsewhere = cache._on(stream)
    assert got == raw
    x = cache._empty((4,), torch.uint8, got, elsewhere)
    assert x.raw == raw and x.recorded == recorded


def test_a_stream_of_another_device_is_refused(cache):
    with pytest.raises(ValueError, match="another device"):
        cache._on(Stream(0x9000, torch.device("cuda", 1)))
    cache._index = 1                       # and so is a cache of another device than the current one
    with pytest.raises(ValueError, match="another device"):
        cache._on(None)
