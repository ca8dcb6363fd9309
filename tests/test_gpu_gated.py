"""The gated feed-forward block on the GPU against the formulas in float64.

Tolerances, from the arithmetic (u = 2^-24): a product's sum of k terms in fp32 is within (k + 8) u
of the sum of their absolute values; bfloat16 results are within 2^-8 of themselves (half a
step at a power of two) on top.  H = act(G) U carries its factors' errors (|act'| <= 1.13) and
32 u (1 + |G|) for the activation, and is rounded, as dG and dU are, before the next product, which
adds their errors times its other operand's absolute values."""
import pytest
import torch

import paper_2607_20548_amd as soap

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
H = 2.0 ** -8
BF = torch.bfloat16


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def act(x, name):
    if name == "silu":
        s = torch.sigmoid(x)
        return x * s, s * (1 + x * (1 - s))
    c = torch.special.ndtr(x)
    return x * c, c + x * torch.exp(-0.5 * x * x) * 0.3989422804014327


def product(a, b, ea=0.0, eb=0.0):
    """a b and its bound, for operands with errors of ea and eb."""
    size = a.abs() @ b.abs()
    return a @ b, (a.shape[1] + 8) * U * size + (ea @ b.abs() if torch.is_tensor(ea) else 0) + (a.abs() @ eb if torch.is_tensor(eb) else 0)


def within(got, want, bound, what):
    if got.dtype == BF:
        bound = bound + H * (want.abs() + bound)
    else:
        bound = bound + 2 * U * want.abs()
    bad = ~((got.double() - want).abs() <= bound + 1e-37)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:3].tolist(), (got.double() - want).abs().max().item())


def make(T, m, n, p, seed, scale=1.0):
    x = (scale * randn(seed, T, m)).to(BF)
    return (x, (m ** -0.5 * randn(seed + 1, m, n)).to(BF), (m ** -0.5 * randn(seed + 2, m, n)).to(BF),
            (n ** -0.5 * randn(seed + 3, n, p)).to(BF), (0.01 * randn(seed + 4, T, p)).to(BF))


def check(x, wg, wu, wd, dy, name="silu", dtype=torch.float32):
    block = soap.GatedFeedForward(wg, wu, wd, activation=name)
    y, gate, up = block.forward(x)
    alone, none, _ = block.forward(x, keep=False)
    assert none is None and torch.equal(alone, y)
    X, G, V, D, Y = (t.double() for t in (x, wg, wu, wd, dy))
    g, eg = product(X, G)
    u, eu = product(X, V)
    within(gate, g, eg, "gate")
    within(up, u, eu, "up")
    a, _ = act(g, name)
    h = a * u
    eh = 1.13 * eg * u.abs() + a.abs() * eu + 32 * U * (1 + g.abs()) * u.abs()
    eh = eh + H * (h.abs() + eh)
    want, bound = product(h, D, eh)
    within(y, want, bound, "y")

    dx, dwg, dwu, dwd = block.backward(dy, x, gate, up, dtype=dtype)
    assert dwg.dtype is (dtype or torch.float32)
    g, u = gate.double(), up.double()
    a, da = act(g, name)
    slope = 32 * U * (1 + g.abs())
    dh, edh = product(Y, D.T)
    h = a * u
    eh = slope * u.abs()
    eh = eh + H * (h.abs() + eh)
    dg, edg = dh * u * da, u.abs() * (edh * 1.13 + dh.abs() * slope)
    edg = edg + H * (dg.abs() + edg)
    du, edu = dh * a, a.abs() * edh + dh.abs() * slope
    edu = edu + H * (du.abs() + edu)
    one, e1 = product(dg, G.T, edg)
    two, e2 = product(du, V.T, edu)
    within(dx, one + two, 2 * (e1 + e2), "dx")
    within(dwg, *product(X.T, dg, 0.0, edg), "dw_gate")
    within(dwu, *product(X.T, du, 0.0, edu), "dw_up")
    within(dwd, *product(h.T, Y, eh.T.contiguous()), "dw_down")


@pytest.mark.parametrize("T,m,n,p", [
    (1, 8, 8, 8), (1, 64, 128, 64), (2, 2048, 512, 1024), (5, 136, 200, 72), (16, 512, 1024, 512), (17, 1000, 264, 328),
    (33, 256, 136, 264), (64, 512, 640, 512), (65, 72, 1032, 520), (127, 256, 256, 128), (130, 128, 384, 136),
    (300, 520, 776, 264), (777, 392, 520, 648), (1025, 256, 512, 256)])
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_sizes(T, m, n, p, name):
    check(*make(T, m, n, p, T + m), name, torch.float32 if name == "silu" else BF)


@pytest.mark.parametrize("T,m,n,p", [(2100, 1032, 2056, 1032), (4104, 1032, 4168, 3592), (3900, 4040, 1032, 4104)])
def test_large(T, m, n, p):
    """Tiles of either size, some of them cut at their ends, in every product."""
    check(*make(T, m, n, p, 3))


@pytest.mark.parametrize("T,m,n,p", [
    (7, 2048, 264, 136), (48, 4096, 136, 72), (64, 72, 8264, 40), (64, 2056, 136, 2600), (66, 136, 4104, 72), (130, 4096, 72, 264),
    (321, 264, 264, 264), (1500, 72, 72, 80), (20000, 64, 40, 72), (200, 2056, 648, 1288), (3, 16, 65536, 24), (70, 24, 65536, 16),
    (5, 2048, 8192, 1024), (40, 4096, 8192, 1032)])
def test_parts_of_k(T, m, n, p):
    """Long sums of few tiles, cut into parts that are added afterwards, and short ones."""
    check(*make(T, m, n, p, T + n), dtype=BF if T % 2 else torch.float32)


def test_views():
    """Rows of x and dy cut out of wider ones, whose other values are no numbers."""
    x, wg, wu, wd, dy = make(70, 136, 264, 72, 5)
    for cut in (8, 24):
        wx, wy = (torch.full((70, t.shape[1] + 2 * cut), float("nan"), device="cuda", dtype=BF) for t in (x, dy))
        wx[:, cut:-cut], wy[:, cut:-cut] = x, dy
        check(wx[:, cut:-cut], wg, wu, wd, wy[:, cut:-cut])


def test_activations_far_out():
    """Gates of hundreds either way, where exp over- and underflows."""
    check(*make(40, 64, 64, 64, 6, scale=200.0), "silu")
    check(*make(40, 64, 64, 64, 6, scale=200.0), "gelu")


@pytest.mark.parametrize("T", [3, 40, 300])
def test_tokens_stay_apart(T):
    """A token that is no number changes no other token's results."""
    x, wg, wu, wd, dy = make(T, 200, 328, 264, 7)
    block = soap.GatedFeedForward(wg, wu, wd)
    y, gate, up = block.forward(x)
    dx = block.backward(dy, x, gate, up)[0]
    bad, dbad = x.clone(), dy.clone()
    bad[1] = float("nan")
    dbad[1] = float("inf")
    y2, gate2, up2 = block.forward(bad)
    dx2 = block.backward(dbad, bad, gate2, up2)[0]
    keep = torch.arange(T, device="cuda") != 1
    assert torch.equal(y2[keep], y[keep]) and torch.equal(dx2[keep], dx[keep])
    assert y2[1].isnan().all()


def test_gradient_against_differences():
    """<gradient, v> of small weights against the difference quotient of the loss in float64: the
    kernel's gradients are within their bfloat16 operands' 3 * 2^-8 of the terms' sizes, the quotient
    within h^2 of the third derivative."""
    x, wg, wu, wd, dy = make(6, 16, 24, 16, 8)
    block = soap.GatedFeedForward(wg, wu, wd)
    _, gate, up = block.forward(x)
    grads = block.backward(dy, x, gate, up)
    leaves = [t.double() for t in (x, wg, wu, wd)]

    def loss(x, wg, wu, wd):
        return ((act(x @ wg, "silu")[0] * (x @ wu)) @ wd * dy.double()).sum()

    for i, got in enumerate(grads):
        v, h = randn(20 + i, *leaves[i].shape).double(), 1e-4
        hi, lo = list(leaves), list(leaves)
        hi[i], lo[i] = leaves[i] + h * v, leaves[i] - h * v
        want = (loss(*hi) - loss(*lo)) / (2 * h)
        size = (got.double().abs() * v.abs()).sum() + 0.01 * dy.double().abs().sum()
        assert abs((got.double() * v).sum() - want) <= 4 * H * size


def test_offsets_past_32_bits():
    """Rows of G, U, H and their gradients past 2^31 elements: the last ones, which alone have gradients,
    as they are by themselves."""
    T, m, n, p, last = 270000, 64, 8192, 72, 100
    x, wg, wu, wd, dy = make(last, m, n, p, 12)
    X, Y = torch.zeros(T, m, device="cuda", dtype=BF), torch.zeros(T, p, device="cuda", dtype=BF)
    X[-last:], Y[-last:] = x, dy
    block = soap.GatedFeedForward(wg, wu, wd)
    y, gate, up = block.forward(X)
    got = block.backward(Y, X, gate, up)
    few, g, u = block.forward(x)
    want = block.backward(dy, x, g, u)
    assert not y[:-last].any() and not got[0][:-last].any()
    # both within their bounds of the same sums: half steps of bfloat16 on either side of both
    for a, b in zip((y[-last:], gate[-last:], up[-last:], got[0][-last:], *got[1:]), (few, g, u, *want)):
        a, b = a.double(), b.double()
        assert (a - b).norm() <= 4 * H * b.norm()


def test_no_tokens():
    x, wg, wu, wd, dy = make(4, 64, 72, 80, 9)
    block = soap.GatedFeedForward(wg, wu, wd)
    y, gate, up = block.forward(x[:0])
    assert y.shape == (0, 80) and gate.shape == (0, 72)
    dx, *dw = block.backward(dy[:0], x[:0], gate, up)
    assert dx.shape == (0, 64) and not any(w.any() for w in dw)


def test_gradients_that_are_not_wanted():
    """The C entry point with single gradients, into a wider dx."""
    T, m, n, p = 50, 64, 136, 72
    x, wg, wu, wd, dy = make(T, m, n, p, 10)
    block = soap.GatedFeedForward(wg, wu, wd)
    _, gate, up = block.forward(x)
    want = block.backward(dy, x, gate, up)
    need = soap.soap_gated_workspace_bytes(T, m, n, p, True)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    for i in range(4):
        out = torch.full((T, m + 16), 7.0, device="cuda", dtype=BF) if i == 0 else torch.full_like(want[i], 7.0)
        dst = [None] * 4
        dst[i] = out[:, 8:] if i == 0 else out
        soap.soap_gated_backward(T, m, n, p, 0, dy, p, x, m, wg, wu, wd, gate, up, dst[0], m + 16, soap.SOAP_F32, *dst[1:],
                                 work, need)
        assert torch.equal(out[:, 8:-8] if i == 0 else out, want[i])
        if i == 0:
            assert (out[:, :8] == 7).all() and (out[:, -8:] == 7).all()


@pytest.mark.parametrize("T", [1, 20, 200])
def test_stream_graph_and_bits(T):
    x, wg, wu, wd, dy = make(T, 256, 520, 264, 11)
    block = soap.GatedFeedForward(wg, wu, wd)

    def run(**kw):
        y, gate, up = block.forward(x, **kw)
        return (y, gate, up, *block.backward(dy, x, gate, up, **kw))

    want = run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = run(stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for i in range(4):
        x.copy_(randn(30 + i, T, 256))
        graph.replay()
        want = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), i


@pytest.mark.parametrize("T", [1, 32, 64, 65, 200])
def test_infinite_hidden_values(T):
    """H, dG and dU past fp32's range are infinite, and so are the sums over them, whatever the number of
    tokens; the other tokens' Y and dX stay as they are."""
    m, n, p = 72, 136, 80
    x, wg, wu, wd, dy = (t.abs() + 0.01 for t in make(T, m, n, p, 14))
    block = soap.GatedFeedForward(wg, wu, wd)
    y, gate, up = block.forward(x)
    dx = block.backward(dy, x, gate, up)[0]
    big, dbig = x.clone(), dy.clone()
    big[0] *= 1e20
    dbig[0] *= 1e22
    y2, gate2, up2 = block.forward(big)
    dx2, *dw = block.backward(dbig, big, gate2, up2)
    inf = float("inf")
    assert (y2[0] == inf).all() and (dx2[0] == inf).all() and all((w == inf).all() for w in dw)
    assert torch.equal(y2[1:], y[1:]) and torch.equal(dx2[1:], dx[1:])


@pytest.mark.parametrize("T", [1, 40])
def test_hidden_values_past_bfloat16(T):
    """A finite H that would round to infinity in bfloat16 stays finite where two are kept."""
    x, wg, wu = (torch.zeros(s, device="cuda", dtype=BF) for s in ((T, 8), (8, 8), (8, 8)))
    x[0, 0], x[0, 1] = 2.0 ** 64, 2.0 ** 55
    wg[0], wu[0], wu[1] = 0.5, 2, -1
    block = soap.GatedFeedForward(wg, wu, 0.25 * torch.eye(8, device="cuda", dtype=BF))
    y, gate, up = block.forward(x)
    h = (2 - 2.0 ** -9) * 2.0 ** 127
    within(y[0], torch.full((8,), 0.25 * h, device="cuda", dtype=torch.float64), 2.0 ** -16 * h, "y")
    dy = torch.zeros(T, 8, device="cuda", dtype=BF)
    dy[0] = 2.0 ** -10
    gate[0], up[0] = 127 / 64 * 2.0 ** 63, 129 / 128 * 2.0 ** 64
    # dU = dH act(G) and H = act(G) U, of the kept G and U
    _, _, dwu, dwd = block.backward(dy, x, gate, up)
    du, h = 2.0 ** -12 * 127 / 64 * 2.0 ** 63, 127 / 64 * 129 / 128 * 2.0 ** 127
    want = torch.zeros(8, 8, device="cuda", dtype=torch.float64)
    want[0], want[1] = 2.0 ** 64 * du, 2.0 ** 55 * du
    within(dwu, want, 2.0 ** -16 * want, "dw_up")
    within(dwd, torch.full((8, 8), h * 2.0 ** -10, device="cuda", dtype=torch.float64), 2.0 ** -16 * h * 2.0 ** -10, "dw_down")


@pytest.mark.parametrize("T", [1, 64, 65, 300])
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_activations_relative(T, name):
    """Gates of -12 to 12, one by one: act(G) and its derivative to their own size.  The function is within
    (x^2 + 24) u of itself (its exponential's argument of up to x^2 / 2, or |x|, is rounded twice; the rest
    are factors near 1 u each), the derivative's two terms within as much of theirs; H, dG and dU keep two
    bfloat16, 2^-16 of themselves, of up to 64 tokens, and one, 2^-8, of more."""
    n = 512
    g = torch.linspace(-12, 12, n, dtype=torch.float64, device="cuda").to(BF)
    wg, wu = torch.zeros(8, n, device="cuda", dtype=BF), torch.zeros(8, n, device="cuda", dtype=BF)
    wg[0], wu[0] = g, 1
    x, dy = torch.zeros(T, 8, device="cuda", dtype=BF), torch.zeros(T, n, device="cuda", dtype=BF)
    x[0, 0], dy[0] = 1, 1
    block = soap.GatedFeedForward(wg, wu, torch.eye(n, device="cuda", dtype=BF), activation=name)
    y, gate, up = block.forward(x)
    assert torch.equal(gate[0], g) and (up[0] == 1).all()
    dx, dwg, dwu, dwd = block.backward(dy, x, gate, up)
    v = g.double()
    a, d = act(v, name)
    if name == "gelu":
        a = 0.5 * v * torch.special.erfc(-v * 0.5 ** 0.5)
        terms = (a / v).abs() + v.abs() * torch.exp(-0.5 * v * v) * 0.3989422804014327
        d = a / v + v * torch.exp(-0.5 * v * v) * 0.3989422804014327
    else:
        s = torch.sigmoid(v)
        terms = s + (a * (1 - s)).abs()
    keep = 2.0 ** -16 if T <= 64 else H
    rel = (v * v + 24) * U
    within(y[0], a, (rel + keep) * a.abs(), "y")
    within(dwd[:, 0], a, (rel + keep) * a.abs(), "dw_down")
    within(dwu[0], a, (rel + keep) * a.abs(), "dw_up")
    within(dwg[0], d, rel * terms + keep * (d.abs() + rel * terms), "dw_gate")


@pytest.mark.parametrize("T", [16, 40])
@pytest.mark.parametrize("m,n,p,name", [
    (64, 8192, 4096, "silu"), (64, 4096, 8264, "gelu"), (2048, 8264, 64, "silu"), (2048, 8264, 64, "gelu"),
    (64, 8264, 4096, "silu"), (64, 8264, 4096, "gelu"), (8264, 2048, 64, "silu")])
def test_weights_past_the_caches(T, m, n, p, name):
    """Few tokens with weights that are loaded past the caches, in every product, with and without parts
    of k."""
    check(*make(T, m, n, p, 15), name, BF)


@pytest.mark.parametrize("T,m,n,p,name,dtype", [
    (8, 64, 512, 2048, "gelu", BF), (77, 176, 8, 928, "gelu", torch.float32), (400, 1000, 2768, 1000, "silu", BF),
    (400, 136, 13200, 8, "silu", torch.float32), (275, 328, 11608, 80, "silu", BF), (4491, 8, 8816, 152, "silu", BF),
    (16427, 8, 80, 16, "gelu", BF), (18712, 136, 224, 16, "gelu", BF), (11019, 8, 1112, 8, "silu", BF),
    (7081, 1344, 8, 32, "silu", BF), (17785, 32, 2280, 152, "silu", torch.float32), (17077, 2656, 72, 56, "silu", BF),
    (16563, 8, 152, 16, "gelu", BF), (15566, 8, 568, 144, "gelu", torch.float32)])
def test_plans(T, m, n, p, name, dtype):
    """Tiles of either size, in parts and whole, more and fewer than compute units, of every product and
    activation, with gradients stored through the caches and past them."""
    check(*make(T, m, n, p, 16), name, dtype)
