"""Layer norm on the GPU against the formula in float64.

Tolerances, set from the arithmetic (u = 2^-24): a value of fp32 output is a sum
of terms of at most the size of |w h| and |b| (forward) or r (|g| + |mean g| +
|h mean(g h)|) (backward), each within a few dozen roundings, taken here as 64 u
of the terms' size, with x's distance from its mean cancelling up to |x| / std
of it; a bfloat16 output is rounded once more, 2^-9 of its value (doubled for a
value next to a rounding boundary)."""
import numpy as np
import pytest
import torch

import paper_2607_20548_amd as soap

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5


def make(rows, cols, dtype, pad=0, off=0, seed=0, scale=1.0, shift=0.3):
    """[rows, cols] inside a tensor that is wider by pad, from column off on."""
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + rows * 31 + cols)
    wide = torch.randn(max(rows, 1), cols + pad + off, generator=g, device="cuda") * scale + shift
    return wide.to(dtype)[:rows, off:off + cols]


def params(cols, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(cols, generator=g, device="cuda") * 0.3 + 1,
            torch.randn(cols, generator=g, device="cuda") * 0.2)


def stats(x):
    x = x.double()
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    return mean, 1 / (var + EPS).sqrt()


def spread(x):
    """max |x| over the standard deviation of each row: what centring cancels."""
    x = x.double()
    return (1 + x.abs().amax(1) * stats(x)[1])[:, None]


def within(got, want, bound, dtype, what):
    got = got.double()
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * want.abs() + 1e-38
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), (got - want).abs().max().item())


def check(x, dy, w, b, dtype):
    norm = soap.LayerNorm(w, b, eps=EPS, cols=x.shape[1])
    y, mean, rstd = norm.forward(x)
    m, r = stats(x)
    h = (x.double() - m[:, None]) * r[:, None]
    one = torch.ones(x.shape[1], device="cuda", dtype=torch.float64)
    wd = w.double() if w is not None else one
    bd = b.double() if b is not None else 0 * one
    assert ((mean.double() - m).abs() <= 64 * U * (x.double().abs().amax(1) + 1e-30)).all()
    assert ((rstd.double() / r - 1).abs() <= 64 * U * spread(x)[:, 0]).all()
    within(y, wd * h + bd, 64 * U * ((wd * h).abs() + wd.abs() * spread(x) + bd.abs()), dtype, "y")
    dx, dw, db = norm.backward(dy, x, mean, rstd)
    # the gradient for the statistics that the call was given
    mg, rg = mean.double()[:, None], rstd.double()[:, None]
    h = (x.double() - mg) * rg
    d = dy.double()
    g = d * wd
    want = rg * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    size = rg * (g.abs().amax(1, keepdim=True) + (1 + h.abs()) * (g * h).abs().mean(1, keepdim=True)
                 + g.abs().mean(1, keepdim=True)) * spread(x)
    within(dx, want, 64 * U * size, dtype, "dx")
    if w is not None:
        terms = (d.abs() * (h.abs() + spread(x))).sum(0)
        within(dw, (d * h).sum(0), 64 * U * terms, torch.float32, "dweight")
    else:
        assert dw is None
    if b is not None:
        within(db, d.sum(0), 64 * U * d.abs().sum(0), torch.float32, "dbias")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [1, 2, 7, 8, 16, 64, 65, 128, 200, 255, 256, 257, 512, 513, 1000, 1024, 2048,
                                  2049, 2303, 4096, 4100, 8192, 8193, 14336, 16384])
def test_widths(cols, dtype):
    for rows in (1, 3, 70):
        x, dy = make(rows, cols, dtype), make(rows, cols, dtype, seed=3, scale=1e-3, shift=0.0)
        check(x, dy, *params(cols), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(5000, 64), (3001, 300), (2049, 768), (1500, 4096), (700, 16384), (20000, 9)])
def test_many_rows(rows, cols, dtype):
    check(make(rows, cols, dtype), make(rows, cols, dtype, seed=5, shift=0.0), *params(cols), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,off", [(8, 0), (1, 0), (0, 1), (8, 8), (3, 5)])
def test_strides_and_alignment(pad, off, dtype):
    for cols in (64, 1000, 4096):
        x = make(33, cols, dtype, pad, off)
        dy = make(33, cols, dtype, off, pad, seed=2)
        check(x, dy, *params(cols), dtype)


def test_without_weight_or_bias():
    w, b = params(300)
    x, dy = make(50, 300, torch.float32), make(50, 300, torch.float32, seed=4)
    check(x, dy, w, None, torch.float32)
    check(x, dy, None, b, torch.float32)
    check(x, dy, None, None, torch.float32)


def test_large_offsets_and_constant_rows():
    x = make(40, 2048, torch.float32, scale=0.01, shift=100.0)
    check(x, make(40, 2048, torch.float32, seed=8), *params(2048), torch.float32)
    x = torch.full((4, 512), 3.0, device="cuda")
    y, mean, rstd = soap.LayerNorm(cols=512, eps=EPS).forward(x)
    assert (y == 0).all() and (mean == 3).all()
    assert torch.allclose(rstd, torch.full_like(rstd, EPS ** -0.5), rtol=1e-6)


@pytest.mark.parametrize("cols", [8, 500, 4096, 16384])
def test_a_bad_row_stays_alone(cols):
    x = make(37, cols, torch.float32)
    norm = soap.LayerNorm(*params(cols), eps=EPS)
    y, mean, rstd = norm.forward(x)
    bad = x.clone()
    bad[5, cols // 2] = float("nan")
    bad[20, 0] = float("inf")
    y2, mean2, rstd2 = norm.forward(bad)
    keep = torch.ones(37, dtype=torch.bool, device="cuda")
    keep[5] = keep[20] = False
    assert torch.equal(y[keep], y2[keep]) and torch.equal(rstd[keep], rstd2[keep])
    assert y2[5].isnan().all() and y2[20].isnan().any()
    dy = make(37, cols, torch.float32, seed=9)
    dx, _, _ = norm.backward(dy, x, mean, rstd)
    dx2, _, _ = norm.backward(dy, bad, mean2, rstd2)
    assert torch.equal(dx[keep], dx2[keep]) and dx2[5].isnan().all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_rows(dtype):
    w, b = params(100)
    norm = soap.LayerNorm(w, b)
    x = torch.empty(0, 100, dtype=dtype, device="cuda")
    y, mean, rstd = norm.forward(x)
    assert y.shape == (0, 100) and mean.shape == (0,)
    dx, dw, db = norm.backward(x, x, mean, rstd)
    assert dx.shape == (0, 100) and (dw == 0).all() and (db == 0).all()


def test_gradient_against_differences():
    rows, cols, step = 3, 24, 1e-5
    x = make(rows, cols, torch.float32, seed=11)
    w, b = params(cols)
    c = make(rows, cols, torch.float32, seed=12)
    norm = soap.LayerNorm(w, b, eps=EPS)
    _, mean, rstd = norm.forward(x)
    dx, dw, db = norm.backward(c, x, mean, rstd)

    def f(x, w, b):
        m, r = stats(x)
        return ((w * (x - m[:, None]) * r[:, None] + b) * c.double()).sum().item()
    X, W, B = x.double(), w.double(), b.double()
    for k, (t, grad) in enumerate([(X, dx), (W, dw), (B, db)]):
        flat = t.reshape(-1)
        for i in range(0, flat.numel(), 5):
            args = [X, W, B]
            up, down = flat.clone(), flat.clone()
            up[i] += step
            down[i] -= step
            args[k] = up.view(t.shape)
            hi = f(*args)
            args[k] = down.view(t.shape)
            diff = (hi - f(*args)) / (2 * step)
            # central differences: step^2 times third derivatives, 1e-16 / step of rounding
            assert abs(grad.reshape(-1)[i].item() - diff) <= 1e-5 * (1 + abs(diff))


def test_offsets_past_32_bits():
    base = torch.empty(2 * (1 << 30) + 1024, dtype=torch.bfloat16, device="cuda")
    x = base.as_strided((3, 512), (1 << 30, 1))
    x.copy_(make(3, 512, torch.bfloat16))
    w, b = params(512)
    y, mean, rstd = soap.LayerNorm(w, b).forward(x)
    y2, mean2, rstd2 = soap.LayerNorm(w, b).forward(x.contiguous())
    assert torch.equal(y, y2) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)


def test_runs_are_the_same_bit_for_bit():
    x, dy = make(5000, 777, torch.bfloat16), make(5000, 777, torch.bfloat16, seed=6)
    norm = soap.LayerNorm(*params(777))
    _, mean, rstd = norm.forward(x)
    first = norm.backward(dy, x, mean, rstd)
    for _ in range(3):
        for a, b in zip(first, norm.backward(dy, x, mean, rstd)):
            assert torch.equal(a, b)


def test_on_a_stream_of_its_own_and_in_a_graph():
    x, dy = make(300, 1024, torch.float32), make(300, 1024, torch.float32, seed=6)
    norm = soap.LayerNorm(*params(1024))
    want = norm.forward(x)
    grads = norm.backward(dy, x, want[1], want[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = norm.forward(x, stream=side)
    got_grads = norm.backward(dy, x, got[1], got[2], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip((*want, *grads), (*got, *got_grads)):
        assert torch.equal(a, b)
    xs, ds = x.clone(), dy.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = norm.forward(xs)
        out_grads = norm.backward(ds, xs, out[1], out[2])
    for k in range(4):
        xs.copy_(x * (1 + k))
        ds.copy_(dy * (2 - k))
        graph.replay()
        torch.cuda.synchronize()
        want = norm.forward(xs)
        grads = norm.backward(ds, xs, want[1], want[2])
        for a, b in zip((*want, *grads), (*out, *out_grads)):
            assert torch.equal(a, b)


def test_classes_refuse_on_the_gpu():
    norm = soap.LayerNorm(*params(64))
    x = make(4, 64, torch.float32)
    with pytest.raises(ValueError):
        norm.forward(make(4, 65, torch.float32))
    with pytest.raises(ValueError):
        norm.forward(make(64, 4, torch.float32).t())
    with pytest.raises(TypeError):
        norm.forward(x.half())
    _, mean, rstd = norm.forward(x)
    with pytest.raises(ValueError):
        norm.backward(x[:3], x, mean, rstd)
    with pytest.raises(ValueError):
        norm.backward(x, x, mean[:3], rstd)
    with pytest.raises(soap.SoapError) as e:
        soap.LayerNorm(cols=64, eps=0.0).forward(x)
    assert e.value.status == soap.SOAP_ERR_HPARAM
    assert np.isfinite(soap.LayerNorm(cols=64).forward(x)[0].cpu().numpy()).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(2100, 9000), (1300, 8192), (9000, 700), (70000, 33), (40001, 250), (5000, 2048)])
def test_workgroups_that_walk_over_rows(rows, cols, dtype):
    check(make(rows, cols, dtype, seed=31), make(rows, cols, dtype, seed=32, shift=0.0), *params(cols), dtype)
