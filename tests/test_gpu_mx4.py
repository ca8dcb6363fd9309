"""MXFP4 quantisation and products on the GPU against the definition in float64.

Quantised values are compared exactly.  A product sums values of few bits in
fp32: each matrix instruction (64 of the summed axis) rounds its part and the
running sum, both at most S = |A| |B|^T, within 2^-23 of it, so the bound is
(2 ceil(K / 64) + 2) 2^-23 S, plus 2^-8 of the value for a bfloat16 result."""
import pytest
import torch

import paper_2607_20548_amd as soap

pytestmark = pytest.mark.gpu
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def randn(*shape, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed * 1009 + sum(shape))
    x = torch.randn(shape, generator=g, device="cuda") * scale
    return x * torch.exp(1.5 * torch.randn((*shape[:-1], 1), generator=g, device="cuda"))


def power(e):
    """2^e in float64, exactly."""
    table = torch.tensor([2.0 ** i for i in range(-200, 201)], dtype=torch.float64, device="cuda")
    return table[e.long() + 200]


def quantised(x):
    """Values of x (last axis) in MXFP4, float64, from the definition."""
    x = x.double()
    k = x.shape[-1]
    b = torch.nn.functional.pad(x, (0, -k % 32)).unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(b).all(-1, keepdim=True)
    e = torch.where((amax > 0) & ~bad, torch.frexp(torch.where(bad, 1.0, amax))[1] - 3, -127).clamp_min(-127)
    a = b.abs() / power(e)
    q = torch.zeros_like(a)
    for code in range(1, 8):
        mid = (LEVELS[code - 1] + LEVELS[code]) / 2
        up = a >= mid if code % 2 == 0 else a > mid
        q = torch.where(up, torch.tensor(LEVELS[code], dtype=torch.float64, device="cuda"), q)
    v = torch.where(bad, torch.nan, torch.copysign(q, b) * power(e))
    return v.flatten(-2)[..., :k]


def same(a, b):
    return torch.equal(torch.nan_to_num(a.double(), nan=12345.0), torch.nan_to_num(b.double(), nan=12345.0))


def check_quantise(x, row_index=None):
    a, b = soap.mx4_quantize(x, along="both", row_index=row_index)
    src = x
    if row_index is not None:
        ok = (row_index >= 0) & (row_index < x.shape[0])
        src = torch.where(ok[:, None], x[row_index.long().clamp(0, x.shape[0] - 1)], torch.zeros_like(x[:1]))
    assert same(a.values(), quantised(src))
    assert same(b.values(), quantised(src.mT))
    assert same(a.values(torch.bfloat16), quantised(src).to(torch.bfloat16))
    for part, along in ((a, "cols"), (b, "rows")):
        one = soap.mx4_quantize(x, along=along, row_index=row_index)
        assert torch.equal(one.data, part.data) and torch.equal(one.scale, part.scale)
        nb = (part.k + 31) // 32          # the padding holds zeros
        assert (part.data[..., 16 * nb:] == 0).all() and (part.scale[..., nb:] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 31), (5, 33), (32, 64), (33, 256), (64, 257), (100, 300),
                                       (129, 512), (257, 130), (300, 1000), (1000, 777), (768, 2048)])
def test_quantise(rows, cols, dtype):
    check_quantise(randn(rows, cols).to(dtype))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,off", [(1, 0), (0, 1), (8, 8), (4, 4), (3, 2)])
def test_quantise_strides(pad, off, dtype):
    for rows, cols in [(40, 96), (70, 260)]:
        wide = randn(rows, cols + pad + off).to(dtype)
        check_quantise(wide[:, off:off + cols])


def test_quantise_batches():
    for shape in [(3, 64, 96), (5, 33, 70), (2, 300, 257)]:
        x = randn(*shape)
        a, b = soap.mx4_quantize(x, along="both")
        assert same(a.values(), quantised(x)) and same(b.values(), quantised(x.mT))


def test_quantise_gathered_rows():
    x = randn(50, 200).bfloat16()
    idx = torch.randint(-1, 50, (333,), device="cuda", dtype=torch.int32)
    idx[7], idx[8], idx[9] = 50, 1 << 30, -(1 << 30)      # not rows of x: zeros
    check_quantise(x, idx)
    check_quantise(x.float()[:, 3:90], idx)
    none = soap.mx4_quantize(x[:0], row_index=torch.full((5,), 3, dtype=torch.int32, device="cuda"))
    assert (none.values() == 0).all()


def test_every_rounding():
    """Blocks whose largest value fixes the scale and whose others are the levels,
    the middles between them and their neighbours, over the whole exponent range."""
    levels = torch.tensor(LEVELS, dtype=torch.float64)
    mids = (levels[1:] + levels[:-1]) / 2
    vals = torch.cat([levels[:7], mids, mids * (1 + 2 ** -20), mids * (1 - 2 ** -20), torch.tensor([5.5, 7.0, 7.999])])
    vals = torch.cat([vals, vals[:32 - vals.numel() % 32]])[:32]
    rows = []
    for e in list(range(-149, 126)):
        for top in (4.0, 6.0, 7.75):
            b = (vals * 2.0 ** e).float()
            b[31] = top * 2.0 ** e
            rows += [b, -b]
    x = torch.stack(rows).cuda()
    check_quantise(x)
    check_quantise(x.bfloat16())


def test_zeros_infinities_and_nan():
    x = randn(40, 128)
    x[3, 40:50] = 0
    x[4] = 0
    x[5, 7] = float("inf")
    x[6, 70] = -float("inf")
    x[7, 127] = float("nan")
    check_quantise(x)
    a = soap.mx4_quantize(x).values()
    assert a[5, :32].isnan().all() and not a[5, 32:].isnan().any() and not a[8:].isnan().any()


def test_empty():
    e = torch.empty(0, 64, device="cuda")
    a, b = soap.mx4_quantize(e, along="both")
    assert a.values().shape == (0, 64) and b.data.shape == (64, 0)
    w = soap.mx4_quantize(randn(20, 64))
    assert soap.mx4_product(a, w).shape == (0, 20)
    out = soap.mx4_product_k(b, b, torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert out.shape == (3, 64, 64) and (out == 0).all()


def bound(av, bv, k, dtype):
    s = av.abs() @ bv.abs().mT
    out = (2 * (-(-k // 64)) + 2) * 2.0 ** -23 * s
    return out + (2.0 ** -8 * (av @ bv.mT).abs() if dtype == torch.bfloat16 else 0)


def close(got, av, bv, dtype, what=""):
    want = av @ bv.mT
    assert got.dtype == dtype
    err = (got.double() - want).abs()
    assert (err <= bound(av, bv, av.shape[-1], dtype)).all(), (what, err.max().item())


PRODUCTS = [(1, 1, 1), (1, 5, 32), (3, 40, 31), (16, 16, 33), (31, 129, 64), (32, 128, 96), (33, 127, 255),
            (64, 256, 256), (65, 300, 257), (128, 128, 512), (130, 513, 1000), (255, 257, 2048), (256, 256, 768),
            (300, 1000, 300), (513, 640, 1056), (1, 2000, 4096), (8, 777, 5000), (1024, 1024, 1024),
            (2049, 515, 416)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product(M, N, K, dtype):
    a, b = soap.mx4_quantize(randn(M, K, seed=1)), soap.mx4_quantize(randn(N, K, seed=2, scale=0.05))
    close(soap.mx4_product(a, b, dtype), a.values().double(), b.values().double(), dtype)


def test_product_into_strided_rows():
    M, N, K = 70, 90, 130
    a, b = soap.mx4_quantize(randn(M, K)), soap.mx4_quantize(randn(N, K, seed=3))
    want = soap.mx4_product(a, b)
    for ld, off, dtype in [(128, 0, torch.float32), (97, 3, torch.float32), (101, 1, torch.bfloat16),
                           (104, 8, torch.bfloat16)]:
        wide = torch.full((M, ld), 7.0, device="cuda", dtype=dtype)
        kind = soap.SOAP_BF16 if dtype == torch.bfloat16 else soap.SOAP_F32
        soap.soap_mx4_gemm(M, N, K, a.data, a.scale, b.data, b.scale, kind,
                           wide.data_ptr() + off * wide.element_size(), ld)
        assert torch.equal(wide[:, off:off + N], want.to(dtype))
        assert (wide[:, :off] == 7).all() and (wide[:, off + N:] == 7).all()


def test_scales_at_the_ends_of_their_range():
    x = randn(64, 128, seed=4) * 2.0 ** -120
    y = randn(64, 128, seed=5) * 2.0 ** 115
    a, b = soap.mx4_quantize(x), soap.mx4_quantize(y)
    close(soap.mx4_product(a, b), a.values().double(), b.values().double(), torch.float32)


def test_nan_reaches_its_row_and_column_only():
    x, y = randn(70, 160), randn(140, 160, seed=6)
    x[5, 40] = float("nan")
    y[9, 0] = float("inf")
    out = soap.mx4_product(soap.mx4_quantize(x), soap.mx4_quantize(y))
    nan = torch.zeros(70, 140, dtype=torch.bool, device="cuda")
    nan[5], nan[:, 9] = True, True
    assert torch.equal(out.isnan(), nan)


def offsets_of(sizes):
    return torch.tensor([0] + list(torch.tensor(sizes).cumsum(0)), dtype=torch.int32, device="cuda")


GROUPS = [([32], 40, 64, 0), ([64, 0, 32, 0, 0, 160], 70, 96, 0), ([0, 0], 33, 64, 64),
          ([32] * 70, 40, 64, 96), ([0] * 65 + [96] + [0] * 3, 128, 256, 0), ([256, 512, 32], 257, 300, 32),
          ([1024, 0, 288], 300, 768, 64), ([32 * (i % 3) for i in range(200)], 64, 128, 320)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,N,K,tail", GROUPS)
def test_product_by_rows(sizes, N, K, tail, dtype):
    M = sum(sizes) + tail
    x, w = randn(M, K, seed=7), randn(len(sizes), N, K, seed=8, scale=0.1)
    x[sum(sizes):] = float("nan")                # rows past the last group are not read
    a, b = soap.mx4_quantize(x), soap.mx4_quantize(w)
    o = offsets_of(sizes)
    got = soap.mx4_product_rows(a, b, o, dtype)
    av, bv = a.values().double(), b.values().double()
    at = 0
    for g, n in enumerate(sizes):
        close(got[at:at + n], av[at:at + n], bv[g], dtype, g)
        at += n
    assert (got[at:] == 0).all()


def test_groups_of_any_number_of_rows():
    sizes, N, K = [1, 7, 0, 33, 129, 2], 50, 70
    M = sum(sizes) + 5
    a, b = soap.mx4_quantize(randn(M, K)), soap.mx4_quantize(randn(len(sizes), N, K, seed=9))
    got = soap.mx4_product_rows(a, b, offsets_of(sizes))
    av, bv, at = a.values().double(), b.values().double(), 0
    for g, n in enumerate(sizes):
        close(got[at:at + n], av[at:at + n], bv[g], torch.float32, g)
        at += n
    assert (got[at:] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,M,N,tail", [([32], 40, 64, 0), ([64, 0, 32, 0, 0, 160], 70, 96, 32),
                                            ([0, 0], 33, 64, 64), ([32] * 70, 40, 50, 0),
                                            ([256, 512, 32], 257, 300, 32), ([1024, 0, 288, 96], 300, 130, 0),
                                            ([32, 2048, 224], 512, 256, 0)])
def test_product_by_k(sizes, M, N, tail, dtype):
    K = sum(sizes) + tail
    x, y = randn(M, K, seed=10), randn(N, K, seed=11, scale=0.01)
    at = 0
    for g, n in enumerate(sizes):                # a group's NaN stays in it
        if g == 1 and n:
            x[3, at] = float("nan")
        at += n
    if tail:
        y[:, at:] = float("nan")
    a, b = soap.mx4_quantize(x), soap.mx4_quantize(y)
    got = soap.mx4_product_k(a, b, offsets_of(sizes), dtype)
    av, bv, at = a.values().double(), b.values().double(), 0
    for g, n in enumerate(sizes):
        part = av[:, at:at + n]
        ok = ~part.isnan().any(1) if n else torch.ones(M, dtype=torch.bool, device="cuda")
        if n:
            close(got[g][ok], part[ok], bv[:, at:at + n], dtype, g)
            assert got[g][~ok].isnan().all()
        else:
            assert (got[g] == 0).all()
        at += n


def test_offsets_outside_the_matrix_stay_inside():
    a, b = soap.mx4_quantize(randn(128, 64)), soap.mx4_quantize(randn(3, 40, 64, seed=12))
    got = soap.mx4_product_rows(a, b, torch.tensor([0, 64, 1 << 30, 1 << 30], dtype=torch.int32, device="cuda"))
    av, bv = a.values().double(), b.values().double()
    close(got[:64], av[:64], bv[0], torch.float32)
    close(got[64:], av[64:], bv[1], torch.float32)
    t = soap.mx4_quantize(randn(40, 128))
    got = soap.mx4_product_k(t, t, torch.tensor([0, 64, 1 << 30, 1 << 30], dtype=torch.int32, device="cuda"))
    tv = t.values().double()
    close(got[0], tv[:, :64], tv[:, :64], torch.float32)
    close(got[1], tv[:, 64:], tv[:, 64:], torch.float32)
    assert (got[2] == 0).all()


def test_offsets_past_32_bits():
    """Packed rows past 2^31 bytes (128 a row), their scales and the outputs past 2^31."""
    rows, k, n = (1 << 24) + 300, 256, 192
    data = torch.zeros(rows, k // 2, dtype=torch.uint8, device="cuda")
    scale = torch.zeros(rows, k // 32, dtype=torch.uint8, device="cuda")
    part = soap.mx4_quantize(randn(300, k, seed=13))
    data[-300:], scale[-300:] = part.data, part.scale
    a = soap.Mx4(data, scale, k)
    b = soap.mx4_quantize(randn(n, k, seed=14))
    got = soap.mx4_product(a, b, torch.bfloat16)
    close(got[-300:], part.values().double(), b.values().double(), torch.bfloat16)
    assert (got[:1000] == 0).all()
    o = torch.tensor([0, 64, rows], dtype=torch.int32, device="cuda")
    two = soap.Mx4(torch.stack([b.data, b.data]), torch.stack([b.scale, b.scale]), k)
    got = soap.mx4_product_rows(a, two, o, torch.bfloat16)
    close(got[-300:], part.values().double(), b.values().double(), torch.bfloat16)
    del got
    vals = a.values(torch.bfloat16)
    assert torch.equal(vals[-300:], part.values(torch.bfloat16))
    again = soap.mx4_quantize(vals)
    assert torch.equal(again.data[-300:], part.data) and torch.equal(again.scale[-300:], part.scale)


def test_the_plan_drives_the_products():
    """Router, gathered rows, products by rows and by k, as a layer uses them."""
    T, E, k, m, n = 300, 12, 3, 160, 96
    x = randn(T, m).bfloat16()
    w = randn(E, m, n, seed=15, scale=0.05)
    r = soap.Router(E, k).forward(randn(T, E, seed=16))
    wt = soap.mx4_quantize(w, along="rows")
    xq = soap.mx4_quantize(x, row_index=r.row_token)
    y = soap.mx4_product_rows(xq, wt, r.offsets)
    xv, wv = quantised(x), quantised(w.mT)
    for t in range(0, T, 17):
        for j in range(k):
            close(y[r.position[t, j]][None], xv[t][None], wv[r.index[t, j]], torch.float32)
    dw = soap.mx4_product_k(soap.mx4_quantize(x, along="rows", row_index=r.row_token),
                            soap.mx4_quantize(y, along="rows"), r.offsets)
    rows, o = r.row_token.long(), r.offsets.tolist()
    xg = torch.where((rows >= 0)[:, None], x.double()[rows.clamp_min(0)], 0.0)
    xt, yt = quantised(xg.mT), quantised(y.mT)
    for e in range(E):
        if o[e + 1] > o[e]:
            close(dw[e], xt[:, o[e]:o[e + 1]], yt[:, o[e]:o[e + 1]], torch.float32, e)


def test_on_a_stream_of_its_own_and_in_a_graph():
    x, w = randn(200, 512).bfloat16(), soap.mx4_quantize(randn(300, 512, seed=17))
    want = soap.mx4_product(soap.mx4_quantize(x), w, torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = soap.mx4_product(soap.mx4_quantize(x, stream=side), w, torch.bfloat16, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    xs = x.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = soap.mx4_quantize(xs, along="both")
        out = soap.mx4_product(a, w, torch.bfloat16)
        vals = b.values()
    for k in range(4):
        xs.copy_(x * (k - 1.5))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, soap.mx4_product(soap.mx4_quantize(xs), w, torch.bfloat16))
        assert torch.equal(vals, soap.mx4_quantize(xs, along="rows").values())


def test_runs_are_the_same_bit_for_bit():
    a, b = soap.mx4_quantize(randn(100, 4096)), soap.mx4_quantize(randn(700, 4096, seed=18))
    first = soap.mx4_product(a, b)
    for _ in range(3):
        assert torch.equal(first, soap.mx4_product(a, b))


def test_classes_refuse_on_the_gpu():
    a, b = soap.mx4_quantize(randn(10, 64)), soap.mx4_quantize(randn(10, 65))
    with pytest.raises(ValueError):
        soap.mx4_product(a, b)
    with pytest.raises(TypeError):
        soap.mx4_product(a, a, torch.float16)
    with pytest.raises(ValueError):
        soap.mx4_product_rows(a, a, torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        soap.mx4_product_k(a, a, torch.zeros(2, device="cuda"))
    with pytest.raises(ValueError):
        soap.mx4_quantize(randn(64, 10).t())
    with pytest.raises(ValueError):
        soap.mx4_quantize(randn(2, 4, 8), row_index=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        a.values(torch.float16)
    with pytest.raises(ValueError):
        soap.Mx4(a.data, a.scale, 300)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(4096, 4096, 300), (3600, 4100, 513), (4096, 3841, 1280), (1000, 1100, 200),
                                   (5000, 700, 256), (700, 5000, 257), (2000, 2100, 640), (16, 16000, 512),
                                   (17, 16001, 300)])
def test_larger_products(M, N, K, dtype):
    """Every tile shape: few rows, 128-tiles with one and two slabs in LDS, 256-tiles."""
    a, b = soap.mx4_quantize(randn(M, K, seed=21)), soap.mx4_quantize(randn(N, K, seed=22, scale=0.05))
    close(soap.mx4_product(a, b, dtype), a.values().double(), b.values().double(), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off", [0, 1])
def test_larger_products_into_strided_rows(dtype, off):
    for M, N, K in [(4096, 4093, 300), (2000, 1001, 640), (1500, 1203, 100)]:
        a, b = soap.mx4_quantize(randn(M, K, seed=23)), soap.mx4_quantize(randn(N, K, seed=24))
        want = soap.mx4_product(a, b, dtype)
        ld = (N + 15) // 8 * 8 if off == 0 else N + 6
        wide = torch.full((M, ld), 7.0, device="cuda", dtype=dtype)
        kind = soap.SOAP_BF16 if dtype == torch.bfloat16 else soap.SOAP_F32
        soap.soap_mx4_gemm(M, N, K, a.data, a.scale, b.data, b.scale, kind,
                           wide.data_ptr() + off * wide.element_size(), ld)
        assert torch.equal(wide[:, off:off + N], want)
        assert (wide[:, :off] == 7).all() and (wide[:, off + N:] == 7).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,N,K,tail", [([700, 0, 900, 33, 5, 2000], 777, 300, 100),
                                            ([32 * (i % 5) for i in range(100)], 520, 256, 64),
                                            ([0] * 70 + [1500, 1, 1, 1], 1000, 130, 0)])
def test_larger_products_by_rows(sizes, N, K, tail, dtype):
    M = sum(sizes) + tail
    x, w = randn(M, K, seed=25), randn(len(sizes), N, K, seed=26, scale=0.1)
    x[sum(sizes):] = float("nan")
    a, b = soap.mx4_quantize(x), soap.mx4_quantize(w)
    got = soap.mx4_product_rows(a, b, offsets_of(sizes), dtype)
    av, bv, at = a.values().double(), b.values().double(), 0
    for g, n in enumerate(sizes):
        close(got[at:at + n], av[at:at + n], bv[g], dtype, g)
        at += n
    assert (got[at:] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_larger_products_by_k(dtype):
    """A gradient larger than the L2s, groups that start and end anywhere in a slab."""
    sizes = [32 * ((7 * i) % 23) for i in range(40)]
    K = sum(sizes) + 32
    a, b = soap.mx4_quantize(randn(640, K, seed=27)), soap.mx4_quantize(randn(700, K, seed=28))
    got = soap.mx4_product_k(a, b, offsets_of(sizes), dtype)
    av, bv, at = a.values().double(), b.values().double(), 0
    for g, n in enumerate(sizes):
        if n:
            close(got[g], av[:, at:at + n], bv[:, at:at + n], dtype, g)
        else:
            assert (got[g] == 0).all()
        at += n


def test_sums_of_a_long_axis():
    """65 536 values of one sign: the running sum is exact to its own last bits."""
    K = 65536
    x = randn(40, K, seed=29).abs()
    a = soap.mx4_quantize(x)
    close(soap.mx4_product(a, a), a.values().double(), a.values().double(), torch.float32)
    b = soap.mx4_quantize(randn(2000, 8192, seed=30).abs())
    close(soap.mx4_product(b, b), b.values().double(), b.values().double(), torch.float32)


@pytest.mark.parametrize("rows,x_rows,k", [(5, 3, 1), (300, 40, 256), (1000, 77, 257), (4096, 512, 4100), (3, 0, 64)])
def test_gathered_packed_rows(rows, x_rows, k):
    x = soap.mx4_quantize(randn(x_rows, k, seed=33))
    idx = torch.randint(-1, max(x_rows, 1), (rows,), device="cuda", dtype=torch.int32)
    idx[0], idx[1] = x_rows, -(1 << 30)
    data = torch.full((rows, x.data.shape[1]), 255, dtype=torch.uint8, device="cuda")
    scale = torch.full((rows, x.scale.shape[1]), 255, dtype=torch.uint8, device="cuda")
    soap.soap_mx4_gather(rows, k, idx, x_rows, x.data, x.scale, data, scale)
    ok = ((idx >= 0) & (idx < x_rows))[:, None]
    at = idx.long().clamp(0, max(x_rows - 1, 0))
    pick = lambda t: torch.where(ok, t[at], torch.zeros_like(t[:1])) if x_rows else torch.zeros_like(data if t is x.data else scale)  # noqa: E731,E501
    assert torch.equal(data, pick(x.data)) and torch.equal(scale, pick(x.scale))


def test_rows_taken_often_are_the_same():
    """Quantised once and copied, or row by row."""
    x = randn(200, 2100, seed=34).bfloat16()
    idx = torch.randint(-1, 200, (17000,), device="cuda", dtype=torch.int32)
    idx[3] = 200
    many = soap.mx4_quantize(x, row_index=idx)
    few = [soap.mx4_quantize(x, row_index=idx[i:i + 1000].contiguous()) for i in range(0, 17000, 1000)]
    assert torch.equal(many.data, torch.cat([f.data for f in few]))
    assert torch.equal(many.scale, torch.cat([f.scale for f in few]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [1, 2, 3, 4, 5, 7, 255, 257, 258, 259, 260, 511, 770])
def test_right_edges_among_nan(cols, dtype):
    """What lies around the matrix, and rows that no index names, are not read into it."""
    full = torch.full((70, cols + 9), torch.nan, device="cuda", dtype=dtype)
    for off in (0, 1, 5):
        x = full[1:67, off:off + cols]
        x.copy_(randn(66, cols, seed=35 + off))
        x[3] = torch.inf
        check_quantise(x)
        idx = torch.tensor([65, -1, 0, 66, 7, 7, -5, 1 << 30] * 9 + [64], device="cuda", dtype=torch.int32)
        check_quantise(x, idx)
        full.fill_(torch.nan)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [250, 300, 700, 1100, 2400, 4200])
def test_values_into_strided_rows(cols, dtype):
    """Every number of lanes a row, rows that start at any element."""
    q = soap.mx4_quantize(randn(37, cols, seed=36))
    want = q.values(torch.float32)
    full = torch.full((37, cols + 5), 7.0, device="cuda", dtype=dtype)
    kind = soap.SOAP_F32 if dtype == torch.float32 else soap.SOAP_BF16
    soap.soap_mx4_dequantize(37, cols, q.data, q.scale, kind, full[:, 3:], full.stride(0))
    assert torch.equal(full[:, 3:3 + cols], want.to(dtype))
    assert (full[:, :3] == 7).all() and (full[:, 3 + cols:] == 7).all()
