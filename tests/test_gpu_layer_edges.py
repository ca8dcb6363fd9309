"""The layer's operators at the edges of their interface, on the GPU."""
import pytest
import torch

import paper_2607_20548_amd as soap
from tests.test_gpu_mx4 import close, offsets_of

pytestmark = pytest.mark.gpu


def randn(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(1013 * seed + sum(shape))
    return torch.randn(shape, generator=g, device="cuda")


# ------------------------------------------------------------------ streams
def cases():
    """name -> (fresh inputs, call(inputs, stream) -> outputs)."""
    norm = soap.LayerNorm(1 + 0.1 * randn(256), 0.1 * randn(256, seed=1))
    router = soap.Router(32, 4)
    w = soap.mx4_quantize(randn(96, 256, seed=2))
    bank = soap.mx4_quantize(randn(2, 96, 256, seed=3))
    offsets = torch.tensor([0, 64, 192], dtype=torch.int32, device="cuda")
    x, dy, l = randn(192, 256, seed=4), randn(192, 256, seed=5), randn(192, 32, seed=6)
    _, mean, rstd = norm.forward(x)
    r = router.forward(l)
    a, at = soap.mx4_quantize(x), soap.mx4_quantize(x, along="rows")
    index = torch.arange(191, -1, -1, dtype=torch.int32, device="cuda")

    def routing(l, stream):
        q = router.forward(l, stream=stream)
        return [getattr(q, name) for name in soap.Routing.__slots__]

    def packed(*ms):
        return [t for m in ms for t in (m.data, m.scale)]
    mx = lambda d, s, k=256: soap.Mx4(d, s, k)  # noqa: E731
    return {
        "norm": ([x], lambda x, stream: norm.forward(x, stream=stream)),
        "norm_grad": ([dy, x, mean, rstd], lambda *t, stream: norm.backward(*t, stream=stream)),
        "route": ([l], routing),
        "route_grad": ([l, r.index, r.counts, r.gate],
                       lambda *t, stream: [router.backward(*t, stream=stream)]),
        "quantize": ([x], lambda x, stream: packed(*soap.mx4_quantize(x, along="both", stream=stream))),
        "gather": ([x, index], lambda x, i, stream: packed(soap.mx4_quantize(x, row_index=i, stream=stream))),
        "values": ([a.data, a.scale], lambda d, s, stream: [mx(d, s).values(stream=stream)]),
        "product": ([a.data, a.scale], lambda d, s, stream: [soap.mx4_product(mx(d, s), w, stream=stream)]),
        "product_rows": ([a.data, a.scale, offsets],
                         lambda d, s, o, stream: [soap.mx4_product_rows(mx(d, s), bank, o, stream=stream)]),
        "product_k": ([at.data, at.scale, offsets],
                      lambda d, s, o, stream: [soap.mx4_product_k(mx(d, s, 192), mx(d, s, 192), o, stream=stream)]),
    }


NAMES = ["norm", "norm_grad", "route", "route_grad", "quantize", "gather", "values", "product", "product_rows",
         "product_k"]


def busy(buffer):
    """Some milliseconds of work on the current stream."""
    for _ in range(20):
        buffer.mul_(1.0)


@pytest.mark.parametrize("how", ["object", "handle", "default"])
@pytest.mark.parametrize("name", NAMES)
def test_a_call_follows_the_work_of_its_stream(name, how):
    """The inputs become right only at the end of long work on the stream that is named;
    the current stream does not wait for it.  Until then they hold other valid values."""
    inputs, call = cases()[name]
    want = call(*inputs, stream=None)
    late = [torch.zeros_like(t) for t in inputs]
    buffer = torch.zeros(1 << 28, device="cuda")
    torch.cuda.synchronize()
    named, current = torch.cuda.Stream(), torch.cuda.Stream()
    if how == "default":
        named = torch.cuda.default_stream()
    with torch.cuda.stream(named):
        busy(buffer)
        for t, v in zip(late, inputs):
            t.copy_(v)
    with torch.cuda.stream(current):
        got = call(*late, stream=named if how == "object" else named.cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b), name


@pytest.mark.parametrize("name", NAMES)
def test_inputs_dropped_after_a_call_are_not_reused_before_it(name):
    """The caller lets go of the inputs while the named stream has yet to read them, and the
    current stream allocates and fills as much."""
    inputs, call = cases()[name]
    want = call(*inputs, stream=None)
    buffer = torch.zeros(1 << 28, device="cuda")
    own = [t.clone() for t in inputs]
    torch.cuda.synchronize()
    named = torch.cuda.Stream()
    with torch.cuda.stream(named):
        busy(buffer)
    got = call(*own, stream=named)
    sizes = [(t.shape, t.dtype) for t in own]
    del own
    taken = [torch.zeros(s, dtype=d, device="cuda") for s, d in sizes for _ in range(2)]
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b), name
    assert taken


# ------------------------------------------------------------ empty token axes
def test_a_router_without_tokens_writes_its_offsets():
    """index, gate, position and row_token are empty then and may be NULL."""
    E = 9
    counts, offsets = (torch.full((E + 1,), 7, dtype=torch.int32, device="cuda") for _ in range(2))
    loss = torch.full((1,), 7.0, device="cuda")
    need = soap.soap_router_workspace_bytes(0, E)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    soap.soap_router_forward(0, E, 2, soap.SOAP_F32, None, E, None, 0, 0.01, None, None, counts, loss, offsets, None,
                             None, ws, need)
    assert (counts == 0).all() and (offsets == 0).all() and loss.item() == 0


@pytest.mark.parametrize("which", ["dweight", "dbias", "both"])
def test_a_layer_norm_without_rows_writes_its_sums(which):
    """The workspace of no rows is empty and may be NULL."""
    cols = 300
    assert soap.soap_layer_norm_workspace_bytes(0, cols) == 0
    dweight, dbias = (torch.full((cols,), 7.0, device="cuda") for _ in range(2))
    soap.soap_layer_norm_backward(0, cols, soap.SOAP_BF16, None, cols, None, cols, None, None, None, None, cols,
                                  None if which == "dbias" else dweight, None if which == "dweight" else dbias,
                                  None, 0)
    assert (dweight == (7 if which == "dbias" else 0)).all() and (dbias == (7 if which == "dweight" else 0)).all()


# ------------------------------------------------------- MXFP4 of empty matrices
@pytest.mark.parametrize("dtype", [None, torch.bfloat16])
def test_an_axis_of_no_values(dtype):
    """What a layer without tokens has along its rows: no values, products that are zeros."""
    a, b = (soap.mx4_quantize(torch.empty(0, n, device="cuda"), along="rows") for n in (40, 70))
    kind = dtype or torch.float32
    assert a.k == 0 and a.values(dtype).shape == (40, 0) and a.values(dtype).dtype == kind
    out = soap.mx4_product(a, b, dtype)
    assert out.shape == (40, 70) and out.dtype == kind and (out == 0).all()
    bank = soap.Mx4(b.data.view(2, 35, 0), b.scale.view(2, 35, 0), 0)
    assert bank.values(dtype).shape == (2, 35, 0)
    o = torch.tensor([0, 32, 40], dtype=torch.int32, device="cuda")
    out = soap.mx4_product_rows(a, bank, o, dtype)
    assert out.shape == (40, 35) and out.dtype == kind and (out == 0).all()
    out = soap.mx4_product_k(a, b, 0 * o, dtype)
    assert out.shape == (2, 40, 70) and out.dtype == kind and (out == 0).all()


def test_empty_batches_sides_and_groups():
    """Matrices of no values in every direction are packed, and their products are empty or
    zeros."""
    for shape in [(0, 8, 64), (3, 0, 64), (3, 8, 0), (8, 0), (0, 0)]:
        x = torch.empty(shape, device="cuda")
        for along in ("cols", "rows"):
            q = soap.mx4_quantize(x, along=along)
            assert q.values().shape == (x if along == "cols" else x.mT).shape
        a, b = soap.mx4_quantize(x, along="both")
        assert a.values().shape == x.shape and b.values().shape == x.mT.shape
    i32 = dict(dtype=torch.int32, device="cuda")
    none = soap.mx4_quantize(torch.empty(5, 0, device="cuda"), row_index=torch.zeros(3, **i32))
    assert none.values().shape == (3, 0)
    a = soap.mx4_quantize(randn(40, 64))
    no_bank = soap.mx4_quantize(torch.empty(0, 16, 64, device="cuda"))
    out = soap.mx4_product_rows(a, no_bank, torch.zeros(1, **i32))      # every row is past the last group
    assert out.shape == (40, 16) and (out == 0).all()
    no_rows = soap.mx4_quantize(torch.empty(0, 64, device="cuda"))
    assert soap.mx4_product(a, no_rows).shape == (40, 0) and soap.mx4_product(no_rows, a).shape == (0, 40)
    assert soap.mx4_product_k(a, a, torch.zeros(1, **i32)).shape == (0, 40, 40)
    assert soap.mx4_product_k(a, no_rows, torch.tensor([0, 32, 64], **i32)).shape == (2, 40, 0)
    with pytest.raises(ValueError, match="offsets"):
        soap.mx4_product_k(a, a, torch.empty(0, **i32))
    with pytest.raises(ValueError, match="offsets"):
        soap.mx4_product_rows(a, no_bank, torch.zeros(2, **i32))


# ---------------------------------------------------- parts of a packed bank
@pytest.mark.parametrize("k", [40, 256, 300, 700, 1200])
def test_one_matrix_of_a_packed_bank(k):
    """Its scales start at any multiple of eight bytes."""
    rows = 37
    bank = soap.mx4_quantize(randn(4, rows, k))
    a = soap.mx4_quantize(randn(50, k, seed=1))
    index = torch.arange(rows + 1, dtype=torch.int32, device="cuda").flip(0)      # one past the end
    for e in range(4):
        part = soap.Mx4(bank.data[e], bank.scale[e], k)
        own = soap.Mx4(bank.data[e].clone(), bank.scale[e].clone(), k)
        assert part.scale.data_ptr() % 8 == 0 and (k > 256 or part.scale.data_ptr() % 16 == 8 * (e % 2))
        for dtype in (torch.float32, torch.bfloat16):
            assert torch.equal(part.values(dtype), own.values(dtype))
            assert torch.equal(soap.mx4_product(a, part, dtype), soap.mx4_product(a, own, dtype))
            assert torch.equal(soap.mx4_product(part, a, dtype), soap.mx4_product(own, a, dtype))
        o = torch.tensor([0, 32, 32, rows, rows], dtype=torch.int32, device="cuda")
        assert torch.equal(soap.mx4_product_rows(part, bank, o), soap.mx4_product_rows(own, bank, o))
        o = o // 32 * 32
        assert torch.equal(soap.mx4_product_k(part, part, o), soap.mx4_product_k(own, own, o))
        got = soap._mx4_empty(a.data, (rows + 1,), k)
        soap.soap_mx4_gather(rows + 1, k, index, rows, part.data, part.scale, got.data, got.scale)
        want = soap._mx4_empty(a.data, (rows + 1,), k)
        soap.soap_mx4_gather(rows + 1, k, index, rows, own.data, own.scale, want.data, want.scale)
        assert torch.equal(got.data, want.data) and torch.equal(got.scale, want.scale)


@pytest.mark.parametrize("k", [40, 300])
def test_quantising_into_one_matrix_of_a_packed_bank(k):
    rows = 37
    x = randn(rows, k, seed=2)
    want = soap.mx4_quantize(x)
    want_t = soap.mx4_quantize(x, along="rows")
    bank, bank_t = soap._mx4_empty(x, (3, rows), k), soap._mx4_empty(x, (3, k), rows)
    for m in (bank, bank_t):
        m.data.fill_(7), m.scale.fill_(7)
    # both in one pass, then each alone
    for e, (d, dt) in enumerate([(True, True), (True, False), (False, True)]):
        ptr = lambda m, on: (m.data[e], m.scale[e]) if on else (None, None)  # noqa: E731
        soap.soap_mx4_quantize(1, rows, k, soap.SOAP_F32, x, k, None, 0, *ptr(bank, d), *ptr(bank_t, dt))
        for m, on, w in ((bank, d, want), (bank_t, dt, want_t)):
            if on:
                assert torch.equal(m.data[e], w.data) and torch.equal(m.scale[e], w.scale)
            else:
                assert (m.data[e] == 7).all() and (m.scale[e] == 7).all()


# ------------------------------------------------- both sides of a choice of tiles
@pytest.mark.parametrize("M,N,K", [(16, 16384, 1280), (16, 16384, 1300), (4, 9600, 1792), (5, 9600, 1792), (1, 9000, 2048),
                                   (8, 16384, 2304), (9, 16384, 2304), (16, 9000, 2816), (16, 9000, 5000),
                                   (3, 9000, 15400), (64, 4096, 600), (65, 4096, 600)])
def test_dense_products_of_few_rows(M, N, K):
    a, b = soap.mx4_quantize(randn(M, K)), soap.mx4_quantize(randn(N, K, seed=1))
    for dtype in (torch.float32, torch.bfloat16):
        close(soap.mx4_product(a, b, dtype), a.values().double(), b.values().double(), dtype)


@pytest.mark.parametrize("tiles,N,K", [(34, 512, 600), (35, 512, 600), (28, 1024, 2900), (29, 1024, 2900),
                                       (12, 2048, 300), (13, 2048, 300), (43, 1024, 2817)])
def test_grouped_products_of_few_rows(tiles, N, K):
    """`tiles` tiles of 32 rows in four groups, one of them without any, one with part of a tile."""
    sizes = [32 * (tiles // 3), 0, 32 * (tiles - tiles // 3 - 2) + 11, 32]
    a, b = soap.mx4_quantize(randn(32 * tiles, K)), soap.mx4_quantize(randn(4, N, K, seed=1))
    av, bv = a.values().double(), b.values().double()
    for dtype in (torch.float32, torch.bfloat16):
        got, at = soap.mx4_product_rows(a, b, offsets_of(sizes), dtype), 0
        for g, n in enumerate(sizes):
            close(got[at:at + n], av[at:at + n], bv[g], dtype, g)
            at += n
        assert (got[at:] == 0).all()


# ------------------------------------------------------- rows taken more than once
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,cols,rows", [(300, 1537, 20010), (300, 1537, 9000), (40, 300, 90000), (5000, 2048, 9000),
                                              (5000, 2048, 20000), (0, 4100, 8000), (1, 8192, 4000), (900, 700, 48000)])
def test_rows_taken_often_and_seldom_are_the_same(tokens, cols, rows, dtype):
    """The binding chooses between quantising a row each time it is taken and copying it."""
    x = randn(tokens, cols + 3).to(dtype)[:, :cols]
    index = torch.randint(-1, tokens + 1, (rows,), device="cuda", dtype=torch.int32)
    got = soap.mx4_quantize(x, row_index=index)
    want = soap._mx4_empty(x, (rows,), cols)
    soap.soap_mx4_quantize(1, rows, cols, soap.SOAP_BF16 if dtype == torch.bfloat16 else soap.SOAP_F32, x, cols + 3,
                           index, tokens, want.data, want.scale, None, None)
    assert torch.equal(got.data, want.data) and torch.equal(got.scale, want.scale)


# ------------------------------------------- the functions of the C names, strided outputs
KIND = {torch.float32: soap.SOAP_F32, torch.bfloat16: soap.SOAP_BF16}


def framed(rows, cols, pad, off, dtype):
    """[rows, cols] inside a wider matrix of sevens, and a check that those stay."""
    wide = torch.full((rows, cols + pad + off), 7.0, device="cuda", dtype=dtype)

    def kept():
        return (wide[:, :off] == 7).all() and (wide[:, off + cols:] == 7).all()
    return wide[:, off:off + cols], kept


FRAMES = [(0, 0), (8, 8), (1, 0), (0, 1), (3, 2)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,off", FRAMES)
@pytest.mark.parametrize("rows,cols", [(37, 100), (37, 1030), (70, 4096), (5, 9001)])
def test_layer_norm_into_strided_rows(rows, cols, pad, off, dtype):
    x, dy = randn(rows, cols).to(dtype), randn(rows, cols, seed=1).to(dtype)
    norm = soap.LayerNorm(1 + 0.1 * randn(cols, seed=2), 0.1 * randn(cols, seed=3))
    y, mean, rstd = norm.forward(x)
    dx, dweight, dbias = norm.backward(dy, x, mean, rstd)
    got, kept = framed(rows, cols, pad, off, dtype)
    soap.soap_layer_norm_forward(rows, cols, KIND[dtype], x, cols, norm.weight, norm.bias, norm.eps, got,
                                 got.stride(0), None, None)
    assert torch.equal(got, y) and kept()
    need = soap.soap_layer_norm_workspace_bytes(rows, cols)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    got, kept = framed(rows, cols, pad, off, dtype)
    dw, db = torch.empty_like(dweight), torch.empty_like(dbias)
    args = (rows, cols, KIND[dtype], dy, cols, x, cols, norm.weight, mean, rstd)
    soap.soap_layer_norm_backward(*args, got, got.stride(0), dw, db, ws, need)
    assert torch.equal(got, dx) and kept() and torch.equal(dw, dweight) and torch.equal(db, dbias)
    got, kept = framed(rows, cols, pad, off, dtype)          # each output alone
    soap.soap_layer_norm_backward(*args, got, got.stride(0), None, None, None, 0)
    assert torch.equal(got, dx) and kept()
    for a, b, want in ((dw, None, dweight), (None, db, dbias)):
        (a if b is None else b).fill_(7)
        soap.soap_layer_norm_backward(*args, None, 0, a, b, ws, need)
        assert torch.equal(a if b is None else b, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,off", FRAMES)
@pytest.mark.parametrize("tokens,experts,k", [(50, 64, 4), (300, 100, 8), (40, 600, 3)])
def test_router_gradient_into_strided_rows(tokens, experts, k, pad, off, dtype):
    l, dgate = randn(tokens, experts).to(dtype), randn(tokens, k, seed=1)
    mask = randn(tokens, seed=2) > -1
    dloss = torch.tensor([0.3], device="cuda")
    for renorm in (True, False):
        router = soap.Router(experts, k, renormalize=renorm, balance=0.1)
        r = router.forward(l, mask)
        want = router.backward(l, r.index, r.counts, dgate, dloss, mask)
        got, kept = framed(tokens, experts, pad, off, dtype)
        soap.soap_router_backward(tokens, experts, k, KIND[dtype], l, experts, mask, router.flags, 0.1, r.index,
                                  r.counts, dgate, dloss, got, got.stride(0))
        assert torch.equal(got, want) and kept()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [1, 8])
def test_quantising_batches_of_strided_rows(pad, dtype):
    batch, rows, cols = 3, 45, 300
    wide = randn(batch, rows, cols + pad).to(dtype)
    x = wide[:, :, :cols].contiguous()
    want, want_t = soap.mx4_quantize(x, along="both")
    got, got_t = soap._mx4_empty(x, (batch, rows), cols), soap._mx4_empty(x, (batch, cols), rows)
    soap.soap_mx4_quantize(batch, rows, cols, KIND[dtype], wide, cols + pad, None, 0, got.data, got.scale, got_t.data,
                           got_t.scale)
    for a, b in ((got, want), (got_t, want_t)):
        assert torch.equal(a.data, b.data) and torch.equal(a.scale, b.scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,off", FRAMES)
@pytest.mark.parametrize("sizes,N,K", [([32, 0, 45], 70, 100), ([700, 0, 900, 33], 777, 300)])
def test_grouped_products_into_strided_rows(sizes, N, K, pad, off, dtype):
    M = sum(sizes) + 20
    a, b = soap.mx4_quantize(randn(M, K)), soap.mx4_quantize(randn(len(sizes), N, K, seed=1))
    o = offsets_of(sizes)
    want = soap.mx4_product_rows(a, b, o, dtype)
    got, kept = framed(M, N, pad, off, dtype)
    soap.soap_mx4_gemm_rows(len(sizes), M, N, K, o, a.data, a.scale, b.data, b.scale, KIND[dtype], got, got.stride(0))
    assert torch.equal(got, want) and kept()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N", [(40, 64), (33, 127)])
def test_products_by_k_at_any_element(M, N, dtype):
    sizes = [64, 0, 96, 32]
    K = sum(sizes)
    a, b, o = soap.mx4_quantize(randn(M, K)), soap.mx4_quantize(randn(N, K, seed=1)), offsets_of(sizes)
    want = soap.mx4_product_k(a, b, o, dtype)
    for off in (0, 1, 8):
        flat = torch.full((4 * M * N + 16,), 7.0, device="cuda", dtype=dtype)
        soap.soap_mx4_gemm_k(4, M, N, K, o, a.data, a.scale, b.data, b.scale, KIND[dtype], flat[off:])
        assert torch.equal(flat[off:off + 4 * M * N].view(4, M, N), want)
        assert (flat[:off] == 7).all() and (flat[off + 4 * M * N:] == 7).all()


def test_sums_over_the_longest_axis():
    """2^25 values a row: a tile's packed rows reach 2^31 bytes.  The second group is the
    last 4096 values but 64."""
    K, M, N = 2 * soap.SOAP_MAX_ROWS, 131, 70
    g = torch.Generator(device="cuda").manual_seed(7)

    def packed(rows):
        data = torch.randint(0, 256, (rows, K // 2), generator=g, device="cuda", dtype=torch.uint8)
        scale = torch.randint(120, 130, (rows, K // 32), generator=g, device="cuda", dtype=torch.uint8)
        return soap.Mx4(data, scale, K)
    a, b = packed(M), packed(N)
    ends = [0, K - 4096, K - 64]
    got = soap.mx4_product_k(a, b, torch.tensor(ends, dtype=torch.int32, device="cuda"))
    part = lambda m, lo, hi: soap.Mx4(m.data[:, lo // 2:hi // 2].contiguous(),  # noqa: E731
                                      m.scale[:, lo // 32:hi // 32].contiguous(), hi - lo).values().double()
    want, size = (torch.zeros(M, N, dtype=torch.float64, device="cuda") for _ in range(2))
    step = 1 << 21
    for lo in range(0, K, step):
        av, bv = part(a, lo, lo + step), part(b, lo, lo + step)
        if lo + step == K:
            last = slice(step - 4096, step - 64)
            close(got[1], av[:, last], bv[:, last], torch.float32)
            av[:, step - 4096:] = 0
        want += av @ bv.t().contiguous()
        size += av.abs() @ bv.abs().t().contiguous()
    assert ((got[0].double() - want).abs() <= (2 * (K // 64) + 2) * 2.0 ** -23 * size).all()
    assert (got[0].double() - want).norm() <= 1e-3 * want.norm()       # random signs: far inside the bound
