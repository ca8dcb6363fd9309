"""The router on the GPU against its definition in float64 (numpy loops for the
choice and the plan: integers, equal exactly).

Tolerances (u = 2^-24): p and gates are quotients of exponentials, each within a
few units of its own rounding (the argument l - max is exact to u |l - max|, at
most about 2^6 here): 256 u relative plus 1e-30.  The loss is a sum of positive
terms: the same relative bound.  dlogits are p times a difference of terms of
the size of max |d|: 256 u p max |d|; a bfloat16 output is rounded once more
(2^-8 of its value)."""
import numpy as np
import pytest
import torch

import paper_2607_20548_amd as soap

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def logits(tokens, experts, dtype=torch.float32, seed=0, pad=0, off=0, scale=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed * 101 + tokens + experts)
    wide = torch.randn(tokens, experts + pad + off, generator=g, device="cuda") * scale
    return wide.to(dtype)[:, off:off + experts]


def choose(l, mask, k):
    """index [T, k] from float64 logits on the host."""
    T, E = l.shape
    index = np.full((T, k), -1, dtype=np.int64)
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        key = np.where(np.isnan(l[t]), -np.inf, l[t])
        order = np.argsort(-key, kind="stable")[:k]
        order = order[key[order] > -np.inf]
        index[t, :len(order)] = order
    return index


def softmax(l):
    with np.errstate(invalid="ignore"):
        e = np.exp(l - np.nanmax(np.where(np.isnan(l), -np.inf, l), axis=1, keepdims=True))
        return e / e.sum(1, keepdims=True)


def forward(l, mask, k, renorm, coef):
    T, E = l.shape
    index = choose(l, mask, k)
    routes = (index >= 0).any(1)
    p = np.zeros((T, E))
    if routes.any():
        p[routes] = softmax(l[routes])
    gate = np.where(index >= 0, np.take_along_axis(p, np.maximum(index, 0), 1), 0.0)
    if renorm:
        with np.errstate(invalid="ignore", divide="ignore"):
            gate = np.where(index >= 0, gate / gate.sum(1, keepdims=True), 0.0)
    counts = np.bincount(index[index >= 0], minlength=E)
    n = int(routes.sum())
    loss = coef * E * (counts / max(1, counts.sum()) * p.sum(0)).sum() / n if n else 0.0
    offsets = np.concatenate([[0], ((counts + 31) // 32 * 32).cumsum()])
    position = np.full((T, k), -1)
    row_token = np.full(soap.soap_router_rows(T, E, k), -1)
    seen = np.zeros(E, dtype=np.int64)
    for t in range(T):
        for j in range(k):
            e = index[t, j]
            if e >= 0:
                position[t, j] = offsets[e] + seen[e]
                row_token[position[t, j]] = t
                seen[e] += 1
    return dict(index=index, gate=gate, counts=np.append(counts, n), loss=np.array([loss]), offsets=offsets,
                position=position, row_token=row_token, p=p)


def check(l, k, renorm=True, mask=None, coef=0.02):
    router = soap.Router(l.shape[1], k, renormalize=renorm, balance=coef)
    r = router.forward(l, mask)
    want = forward(l.double().cpu().numpy(), None if mask is None else mask.cpu().numpy(), k, renorm, coef)
    for name in ("index", "counts", "offsets", "position", "row_token"):
        np.testing.assert_array_equal(getattr(r, name).cpu().numpy(), want[name], err_msg=name)
    for name in ("gate", "loss"):
        got = getattr(r, name).double().cpu().numpy()
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want[name]))
        ok = ~np.isnan(got)
        assert (np.abs(got - want[name])[ok] <= 256 * U * np.abs(want[name])[ok] + 1e-30).all(), name
    return router, r, want


SHAPES = [(1, 1, 1), (1, 8, 2), (2, 64, 8), (7, 5, 5), (127, 60, 6), (128, 64, 8), (129, 64, 8), (300, 65, 3),
          (1000, 128, 8), (513, 129, 7), (777, 256, 4), (500, 257, 8), (300, 512, 8), (200, 513, 32),
          (130, 1000, 16), (90, 1024, 32), (2500, 16, 2)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,experts,k", SHAPES)
def test_forward(tokens, experts, k, dtype):
    l = logits(tokens, experts, dtype)
    g = torch.Generator(device="cuda").manual_seed(tokens)
    mask = torch.rand(tokens, generator=g, device="cuda") > 0.2
    check(l, k, renorm=True)
    check(l, k, renorm=False, mask=mask)


def test_many_chunks():
    # past the most chunks a launch has: each takes more tokens
    check(logits(70000, 24, torch.bfloat16), 2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,off", [(1, 0), (0, 3), (8, 8), (5, 1)])
def test_strides_and_alignment(pad, off, dtype):
    for tokens, experts in [(50, 64), (200, 96), (150, 33)]:
        check(logits(tokens, experts, dtype, pad=pad, off=off), 4)


def test_ties_go_to_the_lowest_index():
    l = torch.zeros(300, 70, device="cuda")
    router, r, _ = check(l, 5)
    assert (r.index == torch.arange(5, device="cuda")).all()
    check(torch.randint(-2, 3, (400, 100), device="cuda").float(), 8)
    check(torch.randint(-1, 2, (400, 40), device="cuda").bfloat16(), 8)
    l = torch.zeros(4, 8, device="cuda")
    l[:, ::2] = -0.0                    # both zeros are one value, whatever their bits
    l[1] = l[1].flip(0)
    check(l, 8)
    check(l, 3)


def test_rows_that_choose_less_or_nothing():
    inf = float("inf")
    l = logits(140, 16)
    l[3] = -inf                         # nothing to choose
    l[7, 2:] = -inf                     # two of four
    l[9, :15] = -inf
    l[11] = torch.finfo(torch.float32).min     # masks of the type's lowest value
    l[12, 1:] = torch.finfo(torch.float32).min
    check(l, 4)
    check(l, 4, renorm=False)
    check(l.bfloat16(), 4)
    mask = torch.zeros(140, dtype=torch.bool, device="cuda")
    _, r, _ = check(l, 4, mask=mask)    # no token routes
    assert r.loss.item() == 0 and (r.row_token == -1).all() and (r.gate == 0).all()
    mask[7] = mask[3] = True
    check(l, 4, mask=mask)


def test_nan_and_infinite_logits():
    l = logits(200, 32)
    l[5, 7] = float("nan")
    l[6] = float("nan")
    router, r, want = check(l, 3)
    assert r.gate[5].isnan().all() and r.loss.isnan().all() and (r.index[6] == -1).all()
    assert (r.gate[6] == 0).all() and not r.gate[7:].isnan().any()
    mask = torch.ones(200, dtype=torch.bool, device="cuda")
    mask[5] = False
    _, r, _ = check(l, 3, mask=mask)
    assert not r.gate.isnan().any() and not r.loss.isnan().any()
    l = logits(40, 32)
    l[2, 4] = float("inf")
    r = soap.Router(32, 3).forward(l)
    assert r.index[2, 0] == 4 and (r.index[2] >= 0).all() and r.gate[2].isnan().all()
    assert not r.gate[3:].isnan().any()


@pytest.mark.parametrize("experts", [1, 64, 1000])
def test_no_tokens(experts):
    router = soap.Router(experts, 1)
    l = torch.empty(0, experts, device="cuda")
    r = router.forward(l)
    assert (r.counts == 0).all() and (r.offsets == 0).all() and r.loss.item() == 0
    assert r.index.shape == (0, 1) and r.row_token.numel() == 0
    assert router.backward(l, r.index, r.counts, r.gate).shape == (0, experts)


def test_without_a_plan_or_loss():
    l = logits(500, 40)
    want = soap.Router(40, 3).forward(l)
    index = torch.empty_like(want.index)
    gate, counts = torch.empty_like(want.gate), torch.empty_like(want.counts)
    n = soap.soap_router_workspace_bytes(500, 40)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    soap.soap_router_forward(500, 40, 3, soap.SOAP_F32, l, 40, None, 1, 0.01, index, gate, counts, None, None, None,
                             None, ws, n)
    assert torch.equal(index, want.index) and torch.equal(gate, want.gate) and torch.equal(counts, want.counts)


def gradient(l, index, counts, dgate, dloss, renorm, coef):
    """dlogits from the formulas in float64 (index -1 rows route nothing)."""
    T, E = l.shape
    routes = (index >= 0).any(1)
    p = np.zeros((T, E))
    p[routes] = softmax(l[routes])
    b = dloss * coef * E * counts[:-1] / max(1, counts[:-1].sum()) / max(1, counts[-1])
    d = np.zeros((T, E))
    chosen = np.zeros((T, E), dtype=bool)
    for t, j in zip(*np.nonzero(index >= 0)):
        d[t, index[t, j]] += dgate[t, j]
        chosen[t, index[t, j]] = True
    if renorm:
        gate = np.where(chosen, p, 0)
        gate = gate / np.maximum(gate.sum(1, keepdims=True), 1e-300)
        out = p * (b - (p * b).sum(1, keepdims=True)) + gate * (d - (gate * d).sum(1, keepdims=True))
        size = p * np.abs(b).max() + gate * np.abs(d).max(1, keepdims=True)
    else:
        out = p * (d + b - (p * (d + b)).sum(1, keepdims=True))
        size = p * np.abs(d + b).max(1, keepdims=True)
    return out * routes[:, None], size * routes[:, None]


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,experts,k", SHAPES)
def test_backward(tokens, experts, k, dtype, renorm):
    pad = tokens % 3
    l = logits(tokens, experts, dtype, seed=2, pad=pad)
    if tokens > 5:
        l[1] = -float("inf")
        l[2, 1:] = -float("inf")
    g = torch.Generator(device="cuda").manual_seed(tokens)
    mask = torch.rand(tokens, generator=g, device="cuda") > 0.2
    router = soap.Router(experts, k, renormalize=renorm, balance=0.03)
    r = router.forward(l, mask)
    dgate = torch.randn(tokens, k, generator=g, device="cuda")
    dgate[r.index < 0] = float("nan")            # not read
    dloss = torch.tensor([0.7], device="cuda")
    got = router.backward(l, r.index, r.counts, dgate, dloss, mask=mask)
    assert got.dtype == dtype
    coef = float(np.float32(0.03)) * float(np.float32(0.7))
    want, size = gradient(l.double().cpu().numpy(), r.index.cpu().numpy(), r.counts.cpu().numpy(),
                          dgate.double().cpu().numpy(), 1.0, renorm, coef)
    got = got.double().cpu().numpy()
    bound = 256 * U * size + 1e-30
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * np.abs(want)
    assert (np.abs(got - want) <= bound).all(), np.abs(got - want).max()


@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(renorm):
    T, E, k, coef, step = 6, 10, 3, 0.5, 1e-6
    l = logits(T, E, seed=5)
    router = soap.Router(E, k, renormalize=renorm, balance=coef)
    r = router.forward(l)
    dgate = torch.randn(T, k, device="cuda")
    got = router.backward(l, r.index, r.counts, dgate).double().cpu().numpy()
    index, counts = r.index.cpu().numpy(), r.counts.cpu().numpy()
    c = dgate.double().cpu().numpy()

    def f(l):
        p = softmax(l)
        gate = np.take_along_axis(p, index, 1)
        if renorm:
            gate = gate / gate.sum(1, keepdims=True)
        return (gate * c).sum() + coef * E * (counts[:-1] / counts[:-1].sum() * p.sum(0)).sum() / T
    x = l.double().cpu().numpy()
    for t in range(T):
        for e in range(E):
            up, down = x.copy(), x.copy()
            up[t, e] += step
            down[t, e] -= step
            diff = (f(up) - f(down)) / (2 * step)
            assert abs(got[t, e] - diff) <= 1e-6 * (1 + abs(diff))


def test_gradient_parts():
    l = logits(300, 48)
    router = soap.Router(48, 4, balance=0.1)
    r = router.forward(l)
    only_loss = router.backward(l, r.index, r.counts)
    zero = router.backward(l, r.index, r.counts, torch.zeros_like(r.gate), torch.ones(1, device="cuda"))
    assert torch.equal(only_loss, zero)
    off = router.backward(l, r.index, r.counts, None, torch.zeros(1, device="cuda"))
    assert (off == 0).all()


def test_runs_are_the_same_bit_for_bit():
    l = logits(9000, 96, torch.bfloat16)
    router = soap.Router(96, 6)
    r = router.forward(l)
    dgate = torch.randn(9000, 6, device="cuda")
    dl = router.backward(l, r.index, r.counts, dgate)
    for _ in range(3):
        q = router.forward(l)
        for name in soap.Routing.__slots__:
            assert torch.equal(getattr(r, name), getattr(q, name)), name
        assert torch.equal(dl, router.backward(l, r.index, r.counts, dgate))


def test_on_a_stream_of_its_own_and_in_a_graph():
    l = logits(1000, 64)
    router = soap.Router(64, 4)
    want = router.forward(l)
    dgate = torch.randn(1000, 4, device="cuda")
    dl = router.backward(l, want.index, want.counts, dgate)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = router.forward(l, stream=side)
    dl2 = router.backward(l, got.index, got.counts, dgate, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for name in soap.Routing.__slots__:
        assert torch.equal(getattr(want, name), getattr(got, name)), name
    assert torch.equal(dl, dl2)
    for tokens in (60, 1000):            # one launch and three
        x = l[:tokens].clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = router.forward(x)
            grad = router.backward(x, out.index, out.counts)
        for k in range(4):
            x.copy_(logits(tokens, 64, seed=20 + k))
            graph.replay()
            torch.cuda.synchronize()
            want = router.forward(x)
            for name in soap.Routing.__slots__:
                assert torch.equal(getattr(want, name), getattr(out, name)), name
            assert torch.equal(grad, router.backward(x, want.index, want.counts))


def test_classes_refuse_on_the_gpu():
    router = soap.Router(16, 2)
    l = logits(10, 16)
    r = router.forward(l)
    with pytest.raises(ValueError):
        router.forward(logits(10, 17))
    with pytest.raises(ValueError):
        router.forward(l, torch.ones(9, dtype=torch.bool, device="cuda"))
    with pytest.raises(TypeError):
        router.forward(l, torch.ones(10, device="cuda"))
    with pytest.raises(TypeError):
        router.backward(l, r.index.long(), r.counts)
    with pytest.raises(ValueError):
        router.backward(l, r.index, r.counts[:-1])
    with pytest.raises(soap.SoapError) as e:
        soap.Router(16, 17).forward(l)
    assert e.value.status == soap.SOAP_ERR_SHAPE
