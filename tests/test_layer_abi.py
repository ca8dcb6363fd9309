"""Argument checks of the layer-norm, router and MXFP4 entry points (no GPU):
every refusal comes before anything is enqueued, with its documented status and
a message; only fake pointers are passed, and only to calls that must fail."""
import pytest

import paper_2607_20548_amd as soap

BASE = 0x7f0000000000
MB = 1 << 24


@pytest.fixture(scope="module")
def L():
    from paper_2607_20548_amd import build
    build.build(force=False)
    return soap.lib()


def P(i, off=0):
    return BASE + i * MB + off


def norm_fwd(L, **o):
    a = dict(rows=8, cols=32, dtype=soap.SOAP_BF16, x=P(0), ldx=32, w=P(1), b=P(2), eps=1e-5, y=P(3),
             ldy=32, mean=P(4), rstd=P(5))
    a.update(o)
    return L.soap_layer_norm_forward(*a.values(), None)


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), soap.SOAP_ERR_SHAPE),
    (dict(rows=soap.SOAP_MAX_ROWS + 1), soap.SOAP_ERR_SHAPE),
    (dict(cols=0), soap.SOAP_ERR_SHAPE),
    (dict(cols=soap.SOAP_MAX_DIM + 1, ldx=1 << 20, ldy=1 << 20), soap.SOAP_ERR_SHAPE),
    (dict(ldx=31), soap.SOAP_ERR_SHAPE),
    (dict(ldy=1 << 31), soap.SOAP_ERR_SHAPE),
    (dict(dtype=2), soap.SOAP_ERR_HPARAM),
    (dict(eps=0.0), soap.SOAP_ERR_HPARAM),
    (dict(eps=float("nan")), soap.SOAP_ERR_HPARAM),
    (dict(x=None), soap.SOAP_ERR_NULL),
    (dict(y=None), soap.SOAP_ERR_NULL),
    (dict(x=P(0, 1)), soap.SOAP_ERR_ALIGN),
    (dict(w=P(1, 2)), soap.SOAP_ERR_ALIGN),
    (dict(y=P(0)), soap.SOAP_ERR_ALIAS),
    (dict(y=P(0, 2 * (7 * 32 + 31))), soap.SOAP_ERR_ALIAS),
    (dict(mean=P(5, 4)), soap.SOAP_ERR_ALIAS),
])
def test_layer_norm_forward_refuses(L, over, code):
    assert norm_fwd(L, **over) == code
    assert soap.soap_last_error() != ""


def norm_bwd(L, **o):
    a = dict(rows=8, cols=32, dtype=soap.SOAP_F32, dy=P(0), lddy=32, x=P(1), ldx=32, w=P(2), mean=P(3),
             rstd=P(4), dx=P(5), lddx=32, dw=P(6), db=P(7), ws=P(8),
             wsb=soap.soap_layer_norm_workspace_bytes(8, 32))
    a.update(o)
    return L.soap_layer_norm_backward(*a.values(), None)


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), soap.SOAP_ERR_SHAPE),
    (dict(lddy=8), soap.SOAP_ERR_SHAPE),
    (dict(lddx=8), soap.SOAP_ERR_SHAPE),
    (dict(dtype=-1), soap.SOAP_ERR_HPARAM),
    (dict(dy=None), soap.SOAP_ERR_NULL),
    (dict(mean=None), soap.SOAP_ERR_NULL),
    (dict(rstd=None), soap.SOAP_ERR_NULL),
    (dict(ws=None), soap.SOAP_ERR_NULL),
    (dict(wsb=0), soap.SOAP_ERR_WORKSPACE),
    (dict(ws=P(8, 8)), soap.SOAP_ERR_ALIGN),
    (dict(dx=P(0)), soap.SOAP_ERR_ALIAS),
    (dict(dw=P(7)), soap.SOAP_ERR_ALIAS),
    (dict(ws=P(1, 16)), soap.SOAP_ERR_ALIAS),
])
def test_layer_norm_backward_refuses(L, over, code):
    assert norm_bwd(L, **over) == code
    assert soap.soap_last_error() != ""


def route_fwd(L, **o):
    t, e, k = o.get("tokens", 16), o.get("experts", 8), o.get("top_k", 2)
    a = dict(tokens=t, experts=e, top_k=k, dtype=soap.SOAP_F32, logits=P(0), ld=max(e, 1), mask=P(1), flags=1,
             balance=0.01, index=P(2), gate=P(3), counts=P(4), loss=P(5), offsets=P(6), position=P(7),
             row_token=P(8), ws=P(9), wsb=soap.soap_router_workspace_bytes(16, 8))
    a.update(o)
    return L.soap_router_forward(*a.values(), None)


@pytest.mark.parametrize("over,code", [
    (dict(tokens=-1), soap.SOAP_ERR_SHAPE),
    (dict(tokens=soap.SOAP_MAX_ROWS + 1), soap.SOAP_ERR_SHAPE),
    (dict(experts=0), soap.SOAP_ERR_SHAPE),
    (dict(experts=1025), soap.SOAP_ERR_SHAPE),
    (dict(top_k=0), soap.SOAP_ERR_SHAPE),
    (dict(top_k=9), soap.SOAP_ERR_SHAPE),
    (dict(experts=64, top_k=33), soap.SOAP_ERR_SHAPE),
    (dict(ld=7), soap.SOAP_ERR_SHAPE),
    (dict(dtype=7), soap.SOAP_ERR_HPARAM),
    (dict(flags=2), soap.SOAP_ERR_HPARAM),
    (dict(balance=-1.0), soap.SOAP_ERR_HPARAM),
    (dict(balance=float("inf")), soap.SOAP_ERR_HPARAM),
    (dict(logits=None), soap.SOAP_ERR_NULL),
    (dict(gate=None), soap.SOAP_ERR_NULL),
    (dict(counts=None), soap.SOAP_ERR_NULL),
    (dict(position=None), soap.SOAP_ERR_NULL),
    (dict(offsets=None), soap.SOAP_ERR_NULL),
    (dict(wsb=0), soap.SOAP_ERR_WORKSPACE),
    (dict(index=P(2, 2)), soap.SOAP_ERR_ALIGN),
    (dict(gate=P(2)), soap.SOAP_ERR_ALIAS),
    (dict(mask=P(2, 5)), soap.SOAP_ERR_ALIAS),
])
def test_router_forward_refuses(L, over, code):
    assert route_fwd(L, **over) == code
    assert soap.soap_last_error() != ""


@pytest.mark.parametrize("over,code", [
    (dict(ldd=3), soap.SOAP_ERR_SHAPE),
    (dict(index=None), soap.SOAP_ERR_NULL),
    (dict(counts=None), soap.SOAP_ERR_NULL),
    (dict(dlogits=None), soap.SOAP_ERR_NULL),
    (dict(dlogits=P(0)), soap.SOAP_ERR_ALIAS),
    (dict(dgate=P(4, 1)), soap.SOAP_ERR_ALIGN),
    (dict(flags=4), soap.SOAP_ERR_HPARAM),
])
def test_router_backward_refuses(L, over, code):
    a = dict(tokens=16, experts=8, top_k=2, dtype=soap.SOAP_F32, logits=P(0), ld=8, mask=P(1), flags=1,
             balance=0.01, index=P(2), counts=P(3), dgate=P(4), dloss=P(5), dlogits=P(6), ldd=8)
    a.update(over)
    assert L.soap_router_backward(*a.values(), None) == code


def test_router_rows():
    assert soap.soap_router_rows(0, 8, 2) == 0
    assert soap.soap_router_rows(1, 8, 2) == 64          # two experts of one row
    assert soap.soap_router_rows(1000, 8, 2) >= 2000 + 7 * 31
    assert soap.soap_router_rows(10, 8, 9) == 0 and soap.soap_router_rows(-1, 8, 2) == 0
    for t, e, k in [(3, 5, 2), (129, 64, 8), (4096, 128, 8)]:
        rows = soap.soap_router_rows(t, e, k)
        assert rows % 32 == 0 and t * k + 31 * min(e, t * k) <= rows < t * k + 31 * min(e, t * k) + 32


@pytest.mark.parametrize("over,code", [
    (dict(batch=0), soap.SOAP_ERR_SHAPE),
    (dict(rows=-1), soap.SOAP_ERR_SHAPE),
    (dict(cols=0), soap.SOAP_ERR_SHAPE),
    (dict(ldx=63), soap.SOAP_ERR_SHAPE),
    (dict(batch=2, index=P(1)), soap.SOAP_ERR_SHAPE),
    (dict(index=P(1), x_rows=-1), soap.SOAP_ERR_SHAPE),
    (dict(dtype=3), soap.SOAP_ERR_HPARAM),
    (dict(x=None), soap.SOAP_ERR_NULL),
    (dict(scale=None), soap.SOAP_ERR_NULL),
    (dict(data_t=P(4)), soap.SOAP_ERR_NULL),
    (dict(data=None, scale=None), soap.SOAP_ERR_NULL),
    (dict(data=P(2, 8)), soap.SOAP_ERR_ALIGN),
    (dict(x=P(0, 1)), soap.SOAP_ERR_ALIGN),
    (dict(data=P(0, 16)), soap.SOAP_ERR_ALIAS),
    (dict(scale=P(2, 64)), soap.SOAP_ERR_ALIAS),
])
def test_mx4_quantize_refuses(L, over, code):
    a = dict(batch=1, rows=8, cols=64, dtype=soap.SOAP_BF16, x=P(0), ldx=64, index=None, x_rows=8, data=P(2),
             scale=P(3), data_t=None, scale_t=None)
    a.update(over)
    assert L.soap_mx4_quantize(*a.values(), None) == code
    assert soap.soap_last_error() != ""


def test_mx4_values_refuse(L):
    f = L.soap_mx4_dequantize
    assert f(-1, 64, P(0), P(1), 0, P(2), 64, None) == soap.SOAP_ERR_SHAPE
    assert f(4, 64, P(0), P(1), 0, P(2), 63, None) == soap.SOAP_ERR_SHAPE
    assert f(4, 64, P(0), P(1), 5, P(2), 64, None) == soap.SOAP_ERR_HPARAM
    assert f(4, 64, None, P(1), 0, P(2), 64, None) == soap.SOAP_ERR_NULL
    assert f(4, 64, P(0), P(1), 0, P(0), 64, None) == soap.SOAP_ERR_ALIAS
    assert f(4, 64, P(0, 4), P(1), 0, P(2), 64, None) == soap.SOAP_ERR_ALIGN


@pytest.mark.parametrize("over,code", [
    (dict(M=-1), soap.SOAP_ERR_SHAPE),
    (dict(N=0), soap.SOAP_ERR_SHAPE),
    (dict(K=0), soap.SOAP_ERR_SHAPE),
    (dict(ldc=7), soap.SOAP_ERR_SHAPE),
    (dict(M=1 << 30, N=1 << 24, ldc=1 << 24), soap.SOAP_ERR_SHAPE),   # more tiles than a launch has
    (dict(dtype=2), soap.SOAP_ERR_HPARAM),
    (dict(ad=None), soap.SOAP_ERR_NULL),
    (dict(C=None), soap.SOAP_ERR_NULL),
    (dict(bs=P(3, 4)), soap.SOAP_ERR_ALIGN),
    (dict(C=P(4, 2)), soap.SOAP_ERR_ALIGN),
    (dict(C=P(1)), soap.SOAP_ERR_ALIAS),
])
def test_mx4_product_refuses(L, over, code):
    a = dict(M=4, N=8, K=64, ad=P(0), as_=P(1), bd=P(2), bs=P(3), dtype=soap.SOAP_F32, C=P(4), ldc=8)
    a.update(over)
    assert L.soap_mx4_gemm(*a.values(), None) == code
    assert soap.soap_last_error() != ""


def test_mx4_grouped_products_refuse(L):
    rows = lambda **o: L.soap_mx4_gemm_rows(*dict(dict(  # noqa: E731
        groups=2, M=4, N=8, K=64, off=P(5), ad=P(0), as_=P(1), bd=P(2), bs=P(3), dtype=0, C=P(4), ldc=8),
        **o).values(), None)
    by_k = lambda **o: L.soap_mx4_gemm_k(*dict(dict(  # noqa: E731
        groups=2, M=4, N=8, K=64, off=P(5), ad=P(0), as_=P(1), bd=P(2), bs=P(3), dtype=0, C=P(4)),
        **o).values(), None)
    for f in (rows, by_k):
        assert f(groups=0) == soap.SOAP_ERR_SHAPE
        assert f(N=0) == soap.SOAP_ERR_SHAPE
        assert f(off=None) == soap.SOAP_ERR_NULL
        assert f(off=P(5, 2)) == soap.SOAP_ERR_ALIGN
        assert f(C=P(5)) == soap.SOAP_ERR_ALIAS
        assert f(dtype=9) == soap.SOAP_ERR_HPARAM
    assert rows(K=0) == soap.SOAP_ERR_SHAPE and rows(ldc=2) == soap.SOAP_ERR_SHAPE
    assert by_k(M=0) == soap.SOAP_ERR_SHAPE and by_k(K=-1) == soap.SOAP_ERR_SHAPE


def test_sizes():
    assert soap.soap_mx4_data_bytes(3, 1) == 3 * 128 and soap.soap_mx4_scale_bytes(3, 1) == 3 * 8
    assert soap.soap_mx4_data_bytes(3, 257) == 3 * 256 and soap.soap_mx4_data_bytes(-1, 4) == 0
    assert soap.soap_layer_norm_workspace_bytes(-1, 4) == 0
    assert soap.soap_layer_norm_workspace_bytes(100, 4096) >= 8 * 4096
    assert soap.soap_router_workspace_bytes(10, 0) == 0
    assert soap.soap_router_workspace_bytes(1 << 20, 64) > 0


def test_tensor_checks_of_the_classes():
    import torch
    with pytest.raises(ValueError):
        soap.LayerNorm()                                   # no width
    with pytest.raises(ValueError):
        soap.LayerNorm(torch.ones(8))                      # not on the GPU
    with pytest.raises(TypeError):
        soap.LayerNorm(torch.ones(8, dtype=torch.float64))
    with pytest.raises(ValueError):
        soap.LayerNorm(cols=8).forward(torch.zeros(2, 8))
    with pytest.raises(ValueError):
        soap.Router(8, 2).forward(torch.zeros(2, 8))
    with pytest.raises(ValueError):
        soap.mx4_quantize(torch.zeros(2, 8), along="diagonal")
    with pytest.raises(ValueError):
        soap.mx4_quantize(torch.zeros(2, 8))
    with pytest.raises(ValueError):
        soap.Mx4(torch.zeros(2, 64, dtype=torch.uint8), torch.zeros(2, 8, dtype=torch.uint8), 64)


def test_mx4_gather_refuses(L):
    f = L.soap_mx4_gather
    assert f(-1, 64, P(0), 4, P(1), P(2), P(3), P(4), None) == soap.SOAP_ERR_SHAPE
    assert f(4, 0, P(0), 4, P(1), P(2), P(3), P(4), None) == soap.SOAP_ERR_SHAPE
    assert f(4, 64, P(0), -4, P(1), P(2), P(3), P(4), None) == soap.SOAP_ERR_SHAPE
    assert f(4, 64, None, 4, P(1), P(2), P(3), P(4), None) == soap.SOAP_ERR_NULL
    assert f(4, 64, P(0), 4, P(1), P(2), P(3), None, None) == soap.SOAP_ERR_NULL
    assert f(4, 64, P(0), 4, P(1), P(2), P(1, 16), P(4), None) == soap.SOAP_ERR_ALIAS
    assert f(4, 64, P(0, 2), 4, P(1), P(2), P(3), P(4), None) == soap.SOAP_ERR_ALIGN
