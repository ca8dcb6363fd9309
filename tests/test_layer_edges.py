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


P8 = [0x7f0000000000 + (i << 24) for i in range(8)]


def test_scales_need_eight_bytes_of_alignment(built):
    """A packed row of up to 256 values has eight bytes of scales: matrices of a bank with an
    odd number of rows start at any multiple of that.  (C overlaps an operand: no call is
    made.)"""
    L = soap.lib()
    o = P8[5]
    for off, code in ((0, soap.SOAP_ERR_ALIAS), (8, soap.SOAP_ERR_ALIAS), (4, soap.SOAP_ERR_ALIGN),
                      (1, soap.SOAP_ERR_ALIGN)):
        s0, s1 = P8[1] + off, P8[3] + off
        for a, b in ((s0, P8[3]), (P8[1], s1)):
            assert L.soap_mx4_gemm(4, 8, 64, P8[0], a, P8[2], b, 0, P8[0], 8, None) == code
            assert L.soap_mx4_gemm_rows(2, 4, 8, 64, o, P8[0], a, P8[2], b, 0, P8[0], 8, None) == code
            assert L.soap_mx4_gemm_k(2, 4, 8, 64, o, P8[0], a, P8[2], b, 0, P8[0], None) == code
            assert L.soap_mx4_gather(4, 64, o, 4, P8[0], a, P8[0], b, None) == code
        assert L.soap_mx4_dequantize(4, 64, P8[0], s0, 0, P8[0], 64, None) == code
        assert L.soap_mx4_quantize(1, 8, 64, 0, P8[0], 64, None, 0, P8[0], s0, None, None, None) == code
        assert L.soap_mx4_quantize(1, 8, 64, 0, P8[0], 64, None, 0, None, None, P8[0], s0, None) == code


@pytest.mark.parametrize("kind", [soap.SOAP_BF16, soap.SOAP_F32])
def test_rows_are_copied_when_they_are_taken_often_and_long(kind):
    often = soap._taken_often
    assert often(1 << 17, 1 << 13, 4096, kind) and often(1 << 20, 1, 2048, kind)
    assert not often(1 << 13, 1 << 13, 4096, kind)          # each row once
    assert not often(100, 4, 16384, kind)                   # two launches cost more than they save
    assert not often(1 << 20, 1 << 10, 256, kind)           # a short row leaves a wave idle
    for cols in (700, 1024, 2048, 8192):                    # once it pays, more rows pay too
        of = [often(rows, 4096, cols, kind) for rows in range(0, 300000, 1000)]
        assert of == sorted(of) and of[-1]
