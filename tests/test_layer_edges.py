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


W = torch.zeros(2, 256)
CALLS = [lambda s: soap.LayerNorm(cols=256).forward(W, stream=s),
         lambda s: soap.LayerNorm(cols=256).backward(W, W, W[:, 0], W[:, 0], stream=s),
         lambda s: soap.Router(256, 2).forward(W, stream=s),
         lambda s: soap.Router(256, 2).backward(W, W, W, stream=s),
         lambda s: soap.mx4_quantize(W, stream=s)]


@pytest.mark.parametrize("call", CALLS)
def test_host_tensors_are_refused_alike_with_and_without_a_stream(call):
    for stream in (None, FakeStream(0x9000), 0x9000, 0):
        with pytest.raises(ValueError, match="must live on the GPU"):
            call(stream)


@pytest.mark.parametrize("stream", [None, FakeStream(0x9000), 0])
def test_other_objects_are_refused_alike_with_and_without_a_stream(stream):
    with pytest.raises(TypeError, match="expected a torch tensor"):
        soap.LayerNorm(cols=4).forward([[1.0, 2.0, 3.0, 4.0]], stream=stream)
    with pytest.raises(TypeError, match="expected a torch tensor"):
        soap.mx4_quantize([[1.0]], stream=stream)
