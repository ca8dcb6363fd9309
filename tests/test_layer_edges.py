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


ROWS = [0, 1, 3, 4, 5, 31, 32, 33, 127, 128, 129, 255, 256, 257, 511, 512, 513, 767, 768, 769, 1023, 1024, 1025,
        1101, 2047, 2048, 2049, 2303, 4096, 4097, 8191, 8192, 8193, 16383, 16384, 16385, 32768, 65536, 65537,
        1 << 20, 1 << 24]
WIDTHS = [1, 64, 65, 256, 257, 1000, 2048, 2049, 2303, 4096, 4097, 8191, 8192, 8193, 14336, 16384]


@pytest.fixture(scope="module")
def built():
    from paper_2607_20548_amd import build
    build.build(force=False)
    soap.lib()


def test_a_workspace_of_the_largest_call_is_enough_for_the_others(built):
    """The sizes never shrink as a call grows, in rows or in width."""
    size = soap.soap_layer_norm_workspace_bytes
    for cols in WIDTHS:
        of = [size(rows, cols) for rows in [*range(2600), *(r for r in ROWS if r >= 2600)]]
        assert of == sorted(of), cols
    for rows in ROWS:
        of = [size(rows, cols) for cols in WIDTHS]
        assert of == sorted(of), rows
    size = soap.soap_router_workspace_bytes
    for experts in (1, 8, 64, 1000, 1024):
        of = [size(tokens, experts) for tokens in ROWS]
        assert of == sorted(of), experts
    for tokens in ROWS:
        of = [size(tokens, experts) for experts in range(1, 1025)]
        assert of == sorted(of), tokens
