"""Heads' norm and rotation on the GPU against the formula in float64.

Tolerances, from the arithmetic (u = 2^-24): 1 / sqrt of the mean square of a head is within
24 u (at most 16 products summed in turn by a lane, a tree of 6, division and root); a value of a
pair is then at most four rounded products of |w x r| each, taken as 64 u of the pair's size.  An
angle of t radians is formed in fp64: 2^-51 t, and rounded in half turns: 4 u.  A gradient's terms
|g w| and |h| mean |g w h| are within 96 u each (a second sum over the head), a weight's gradient
adds up to tokens heads / 256 terms in turn.  A bfloat16 output is rounded once more, 2^-8 of its
value with the half step on either side of a power of two."""
import pytest
import torch

import paper_2607_20548_amd as soap

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-6


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def frequencies(rotary, base=10000.0):
    return base ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / max(rotary, 1))


def turn(y, pos, freq, near, back=False):
    """The pairs of float64 heads turned by pos * freq."""
    r = 2 * freq.numel()
    t, rest = y[..., :r], y[..., r:]
    a, b = (t[..., 0::2], t[..., 1::2]) if near else (t[..., :r // 2], t[..., r // 2:])
    angle = pos.double()[:, None, None] * freq * (-1 if back else 1)
    c, s = angle.cos(), angle.sin()
    x, z = a * c - b * s, b * c + a * s
    t = torch.stack([x, z], -1).flatten(-2) if near else torch.cat([x, z], -1)
    return torch.cat([t, rest], -1)


def pair_size(v, rotary, near):
    """|a| + |b| at both values of each pair."""
    v = v.abs()
    t, rest = v[..., :rotary], v[..., rotary:]
    if near:
        s = (t[..., 0::2] + t[..., 1::2]).repeat_interleave(2, -1)
    else:
        s = (t[..., :rotary // 2] + t[..., rotary // 2:]).repeat(*([1] * (v.dim() - 1)), 2)
    return torch.cat([s, rest], -1)


def within(got, want, bound, what):
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (want.abs() + bound) + 1e-38
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), (got.double() - want).abs().max().item())


def check(q, k, wq, wk, pos, freq, near, dq=None, dk=None, dim=None):
    dim = dim or (q if q is not None else k).shape[-1]
    norm = soap.HeadNorm(dim, wq, wk, eps=EPS, frequencies=freq, interleaved=near)
    tokens = (q if q is not None else k).shape[0]
    at = pos if pos is not None else torch.arange(tokens, device="cuda")
    rot = 2 * freq.numel()
    far = 2.0 ** -51 * at.abs().max().double() * (freq.max() if rot else 0) if tokens else 0
    out = norm.forward(q, k, pos)
    grads = norm.backward(dq, dk, q, k, pos) if dq is not None or dk is not None else None
    for i, (x, w, y, d) in enumerate(((q, wq, out[0], dq), (k, wk, out[1], dk))):
        if x is None:
            assert y is None
            continue
        assert y.shape == x.shape and y.dtype == x.dtype and y.is_contiguous()
        xd = x.double()
        wd = w.double() if w is not None else torch.ones(dim, dtype=torch.float64, device="cuda")
        r = 1 / (xd.square().mean(-1, keepdim=True) + EPS).sqrt()
        h = xd * r
        size = pair_size(h * wd, rot, near)
        within(y, turn(h * wd, at, freq, near), (64 * U + far) * size + 1e-38, "y")
        if d is None:
            continue
        dd = d.double()
        g = turn(dd, at, freq, near, back=True)
        gs = pair_size(dd, rot, near) * (1 + far / U / 16)
        dot = (g * wd * h).mean(-1, keepdim=True)
        sizes = r * (gs * wd.abs() + h.abs() * (gs * wd.abs() * h.abs()).mean(-1, keepdim=True))
        within(grads[i], r * (g * wd - h * dot), 96 * U * sizes + 1e-38, "dx")
        if w is None:
            assert grads[2 + i] is None
        else:
            terms = (gs * h.abs()).sum((0, 1))
            n = tokens * x.shape[1] / 256
            within(grads[2 + i], (g * h).sum((0, 1)), (96 + n) * U * terms + 1e-38, "dw")


SIZES = [  # tokens, query heads, key heads, dim, rotary
    (1, 16, 16, 128, 128), (3, 1, 1, 2, 2), (5, 7, 3, 80, 40), (257, 4, 1, 64, 64), (33, 9, 2, 96, 96),
    (64, 2, 2, 256, 256), (7, 3, 5, 18, 6), (2, 5, 4, 512, 512), (9, 2, 3, 510, 2), (4, 64, 8, 128, 64),
    (11, 3, 2, 112, 0), (600, 12, 4, 128, 128), (5000, 3, 1, 32, 32), (13, 2, 1, 34, 34), (6, 17, 0, 128, 128),
    (1001, 1, 1, 128, 64), (77, 3, 1, 256, 256), (130, 1, 0, 64, 64), (65, 5, 3, 24, 12)]


@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,hq,hk,dim,rot", SIZES)
def test_sizes(tokens, hq, hk, dim, rot, dtype, near):
    seed = tokens * 131 + dim
    q = randn(seed, tokens, hq, dim).to(dtype)
    k = (3 * randn(seed + 1, tokens, hk, dim) + 0.2).to(dtype) if hk else None
    wq, wk = 1 + 0.3 * randn(seed + 2, dim), 1 + 0.3 * randn(seed + 3, dim)
    pos = torch.randint(0, 100000, (tokens,), device="cuda", dtype=torch.int32)
    check(q, k, wq, wk, pos, frequencies(rot), near, (1e-3 * randn(seed + 4, tokens, hq, dim)).to(dtype),
          (1e-2 * randn(seed + 5, tokens, hk, dim)).to(dtype) if hk else None)


@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,hq,hk,dim", [
    (50, 32, 32, 64), (50, 32, 32, 32), (50, 16, 16, 64), (20, 4, 4, 256), (20, 8, 8, 256), (30, 2, 2, 512)])
def test_heads_side_by_side(tokens, hq, hk, dim, dtype, near):
    """Heads that fill a wave's slots, and tokens that do, for each number of lanes."""
    q, k, dq, dk = (0.1 + randn(i, tokens, h, dim).to(dtype) for i, h in ((1, hq), (2, hk), (3, hq), (4, hk)))
    check(q, k, 1 + 0.2 * randn(5, dim), 1 + 0.2 * randn(6, dim), None, frequencies(dim), near, dq, dk)


@pytest.mark.parametrize("tokens,hq,hk,dim,dtype", [
    (4001, 22, 14, 128, torch.float32), (8001, 20, 13, 128, torch.bfloat16), (2001, 20, 13, 256, torch.float32),
    (4001, 20, 13, 256, torch.bfloat16), (601, 40, 26, 512, torch.float32), (2001, 20, 13, 512, torch.bfloat16),
    (8001, 20, 13, 64, torch.float32)])
def test_more_than_caches_hold(tokens, hq, hk, dim, dtype):
    """Sizes that are loaded past the caches."""
    q, k, dq, dk = (0.1 + randn(i, tokens, h, dim).to(dtype) for i, h in ((1, hq), (2, hk), (3, hq), (4, hk)))
    wq, wk = 1 + 0.2 * randn(5, dim), 1 + 0.2 * randn(6, dim)
    check(q, k, wq, wk, None, frequencies(dim), False, dq, dk)


def test_more_than_caches_hold_of_short_heads():
    """The smallest halves of whole lines: 32 values of fp32."""
    q, k, dq, dk = (0.1 + randn(i, 8001, 16, 64) for i in range(1, 5))
    check(q, k, 1 + 0.2 * randn(5, 64), 1 + 0.2 * randn(6, 64), None, frequencies(64), False, dq, dk)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_views(dtype):
    """A fused row, rows at odd elements, heads in front of tokens, gradients that repeat."""
    T, dim = 37, 48
    row = randn(3, T, 9 * dim + 1).to(dtype)[:, 1:].view(T, 9, dim)
    w = 1 + 0.1 * randn(4, dim)
    f = frequencies(dim)
    pos = torch.arange(T, device="cuda", dtype=torch.int32) - 5
    d = randn(5, 1, 1, dim).to(dtype)
    check(row[:, :4], row[:, 4:6], w, None, pos, f, False, d.expand(T, 4, dim), d.expand(T, 2, dim))
    heads_first = randn(6, 4, T, dim).to(dtype).transpose(0, 1)
    check(heads_first, None, w, None, None, f, True, randn(7, 4, T, dim).to(dtype).transpose(0, 1))
    check(None, heads_first, None, w, None, f, False, None, heads_first)


def test_extremes():
    """Zero heads, constants, huge and tiny values, far and negative positions, NaN in one head only."""
    dim, f = 64, frequencies(64)
    q = randn(1, 6, 2, dim)
    q[0] = 0
    q[1] = 1e18
    q[2] *= 1e-20
    q[3] *= 1e15
    pos = torch.tensor([0, 1, -7, 2 ** 31 - 1, -2 ** 31, 131071], dtype=torch.int32, device="cuda")
    check(q, q.clone(), None, torch.full((dim,), 2.0, device="cuda"), pos, f, False, randn(2, 6, 2, dim),
          randn(3, 6, 2, dim))
    bad = q.clone()
    bad[4, 1, 3] = float("nan")
    bad[5, 0, 60] = float("inf")
    norm = soap.HeadNorm(dim, frequencies=f, eps=EPS)
    want, got = norm.forward(q, None, pos)[0], norm.forward(bad, None, pos)[0]
    assert got[4, 1].isnan().all() and not got[5, 0].isfinite().all()
    keep = torch.ones(6, 2, dtype=torch.bool, device="cuda")
    keep[4, 1] = keep[5, 0] = False
    assert torch.equal(got[keep], want[keep])


@pytest.mark.parametrize("near", [False, True])
def test_gradient_against_differences(near):
    """<gradient, v> against the difference quotient of the kernel's own forward pass: the step 2^-5
    leaves h^2 of the third derivative (heads of unit values: below 4 h^2 of the direction's
    size) and 64 u / h of rounding."""
    T, H, dim = 3, 2, 32
    f, pos = frequencies(dim), torch.tensor([0, 5, 90000], dtype=torch.int32, device="cuda")
    w, c, x, v = 1 + 0.2 * randn(1, dim), randn(2, T, H, dim), randn(3, T, H, dim), randn(4, T, H, dim)
    vw = randn(5, dim)

    def total(x, w):
        return (soap.HeadNorm(dim, w, eps=EPS, frequencies=f, interleaved=near).forward(x, None, pos)[0].double() * c).sum()

    dx, _, dw, _ = soap.HeadNorm(dim, w, eps=EPS, frequencies=f, interleaved=near).backward(c, None, x, None, pos)
    h = 2.0 ** -5
    size = (c.abs() * 4).sum().item()
    for got, lo, hi in (((dx.double() * v).sum(), (x - h * v, w), (x + h * v, w)),
                        ((dw.double() * vw).sum(), (x, w - h * vw), (x, w + h * vw))):
        want = (total(*hi) - total(*lo)) / (2 * h)
        assert abs(got - want).item() <= (4 * h * h + 64 * U / h) * size


def test_offsets_past_32_bits():
    """Heads past 2^31 elements: the last tokens' as they are by themselves."""
    T, heads, dim, last = 135000, 128, 128, 10
    q = torch.ones(T, heads, dim, device="cuda", dtype=torch.bfloat16)
    dq = torch.zeros_like(q)
    q[-last:], dq[-last:] = randn(1, last, heads, dim), randn(2, last, heads, dim)
    at = torch.arange(T, device="cuda", dtype=torch.int32)
    norm = soap.HeadNorm(dim, 1 + 0.1 * randn(3, dim))
    y, _ = norm.forward(q, None, at)
    dx, _, dw, _ = norm.backward(dq, None, q, None, at)
    args = q[-last:].contiguous(), None, at[-last:].contiguous()
    want = norm.backward(dq[-last:].contiguous(), None, *args)
    assert torch.equal(y[-last:], norm.forward(*args)[0]) and torch.equal(dx[-last:], want[0])
    assert not dx[:-last].any() and (dw - want[2]).norm() <= 2.0 ** -18 * want[2].norm()


def test_no_heads():
    """A side of no heads beside one that has some, and two of none: weights' gradients of zeros."""
    norm = soap.HeadNorm(32, torch.ones(32, device="cuda"), torch.ones(32, device="cuda"))
    none, k = torch.empty(9, 0, 32, device="cuda"), randn(1, 9, 3, 32)
    y, yk = norm.forward(none, k)
    assert y.shape == none.shape and torch.equal(yk, norm.forward(None, k)[1])
    dq, dk, dwq, dwk = norm.backward(none, k, none, k)
    assert dq.shape == none.shape and not dwq.any() and torch.equal(dwk, norm.backward(None, k, None, k)[3])
    _, _, dwq, dwk = norm.backward(none, none, none, none)
    assert not dwq.any() and not dwk.any()


def test_no_tokens():
    norm = soap.HeadNorm(32, torch.ones(32, device="cuda"), torch.ones(32, device="cuda"))
    q, k = torch.empty(0, 4, 32, device="cuda"), torch.empty(0, 2, 32, device="cuda")
    a, b = norm.forward(q, k)
    assert a.shape == q.shape and b.shape == k.shape
    dq, dk, dwq, dwk = norm.backward(q, k, q, k)
    assert dq.shape == q.shape and not dwq.any() and not dwk.any()


def test_output_into_a_fused_row():
    """The C entry point with both gradients written into one row of queries, keys and values, the
    values' part left as it was; overlapping parts are refused."""
    T, hq, hk, dim = 50, 3, 2, 40
    row, out = randn(1, T, 7, dim).bfloat16(), torch.full((T, 7, dim), 7.0, device="cuda", dtype=torch.bfloat16)
    dy = randn(2, T, 5, dim).bfloat16()
    f, wide = frequencies(dim), 7 * dim
    norm = soap.HeadNorm(dim, frequencies=f, eps=EPS)
    want = norm.backward(dy[:, :hq], dy[:, hq:], row[:, :hq], row[:, hq:5])

    def call(dk):
        soap.soap_head_norm_backward(T, hq, hk, dim, dim, soap.SOAP_BF16, 0, dy, 5 * dim, dim, dy[:, hq:], 5 * dim, dim,
                                     row, wide, dim, row[:, hq:], wide, dim, None, None, EPS, None, f, out, wide, dim,
                                     dk, wide, dim, None, None, None, 0)

    call(out[:, hq:])
    assert torch.equal(out[:, :hq], want[0]) and torch.equal(out[:, hq:5], want[1]) and (out[:, 5:] == 7).all()
    with pytest.raises(soap.SoapError) as e:
        call(out[:, hq - 1:])
    assert e.value.status == soap.SOAP_ERR_ALIAS


def test_stream_graph_and_bits():
    """A stream of one's own, a graph replayed with eager work between, the same bits each time."""
    T, H, dim = 700, 5, 64
    f = frequencies(dim)
    w = 1 + 0.1 * randn(1, dim)
    norm = soap.HeadNorm(dim, w, w, eps=EPS, frequencies=f)
    q, k, dq, dk = (randn(i, T, H, dim).bfloat16() for i in range(2, 6))
    pos = torch.arange(T, device="cuda", dtype=torch.int32)
    want = (*norm.forward(q, k, pos), *norm.backward(dq, dk, q, k, pos))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = (*norm.forward(q, k, pos, stream=s), *norm.backward(dq, dk, q, k, pos, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = (*norm.forward(q, k, pos), *norm.backward(dq, dk, q, k, pos))
    for i in range(4):
        q.copy_(randn(20 + i, T, H, dim))
        graph.replay()
        want = (*norm.forward(q, k, pos), *norm.backward(dq, dk, q, k, pos))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), i


def test_built_on_another_stream():
    """Default frequencies are there once the object is: built on a busy stream and used at once on another
    that has waited for nothing, with inputs that were ready before."""
    q, w = randn(1, 300, 4, 64), 1 + 0.1 * randn(2, 64)
    want = soap.HeadNorm(64, w).forward(q)[0]
    x = randn(3, 4096, 4096)
    busy, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(3):
        with torch.cuda.stream(busy):
            for _ in range(20):
                x = (x @ x) * 1e-3
            # what the allocator may hand the frequencies holds other values
            stale = torch.full((32,), 7.0 + i, dtype=torch.float64, device="cuda")
            del stale
            norm = soap.HeadNorm(64, w)
        got = norm.forward(q, stream=other)[0]
        torch.cuda.synchronize()
        assert torch.equal(got, want), i


def test_built_in_a_graph():
    """An object built while a graph is captured, its frequencies part of the graph."""
    q, w = randn(1, 30, 4, 64), 1 + 0.1 * randn(2, 64)
    soap.HeadNorm(64, w).forward(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = soap.HeadNorm(64, w).forward(q)[0]
    for i in range(3):
        q.copy_(randn(5 + i, 30, 4, 64))
        graph.replay()
        want = soap.HeadNorm(64, w).forward(q)[0]
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


def test_heads_in_turn():
    """The C entry points with inputs and outputs of rows in which heads of queries and keys take turns,
    and of one key's between the queries'."""
    T, h, dim = 37, 3, 24
    f = frequencies(dim)
    norm = soap.HeadNorm(dim, frequencies=f, eps=EPS)
    row, dy = randn(1, T, h, 3, dim), randn(2, T, h, 3, dim)
    t, s = 3 * h * dim, 3 * dim
    want = norm.forward(row[:, :, 0], row[:, :, 1])
    dwant = norm.backward(dy[:, :, 0], dy[:, :, 1], row[:, :, 0], row[:, :, 1])
    for kh in (h, 1):
        out, dout = torch.full_like(row, 7.0), torch.full_like(row, 7.0)
        soap.soap_head_norm_forward(T, h, kh, dim, dim, soap.SOAP_F32, 0, row, t, s, row[:, :, 1], t, s, None, None, EPS, None,
                                    f, out, t, s, out[:, :, 1], t, s)
        soap.soap_head_norm_backward(T, h, kh, dim, dim, soap.SOAP_F32, 0, dy, t, s, dy[:, :, 1], t, s, row, t, s,
                                     row[:, :, 1], t, s, None, None, EPS, None, f, dout, t, s, dout[:, :, 1], t, s, None, None,
                                     None, 0)
        for o, w in ((out, want), (dout, dwant)):
            assert torch.equal(o[:, :, 0], w[0]) and torch.equal(o[:, :kh, 1], w[1][:, :kh])
            assert (o[:, kh:, 1] == 7).all() and (o[:, :, 2] == 7).all()
