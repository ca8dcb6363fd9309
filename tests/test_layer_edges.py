"""The binding and the host side of the layer's operators at their edges (no GPU)."""
import contextlib
import types

import pytest
import torch

import paper_2607_20548_amd as soap


class FakeStream:
    def __init__(self, handle):
        self.cuda_stream = handle


def fake_torch(ran):
    """What the binding asks of torch to change streams: a handle of 0 makes torch.cuda.ExternalStream
    take a stream from its pool, the default stream has the handle 0."""
    @contextlib.contextmanager
    def on(stream):
        ran.append(stream.cuda_stream)
        yield
    cuda = types.SimpleNamespace(ExternalStream=lambda h: FakeStream(h or 0x5151), stream=on,
                                 default_stream=lambda: FakeStream(0), Stream=FakeStream)
    return types.SimpleNamespace(cuda=cuda, Tensor=torch.Tensor)


@pytest.mark.parametrize("given,used", [(0, 0), (0x7000, 0x7000), (FakeStream(0x8000), 0x8000), (FakeStream(0), 0)])
def test_a_raw_stream_is_the_one_that_is_used(monkeypatch, given, used):
    ran = []
    monkeypatch.setattr(soap, "_torch", fake_torch(ran))
    assert soap._on(given, (None, None), lambda: "done") == "done"
    assert ran == [used]
