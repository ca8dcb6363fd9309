"""Distillation on the GPU against the formula in float64.

Tolerances, from the arithmetic (u = 2^-24).  An exponential's argument (z - m) / tau is within 3 u
of itself, so the sum of exponentials is within (classes / 512 + 64) u: up to classes / 512 terms
added in turn by a thread, a tree, and d e^-d <= 1 of the arguments' part; its log and a
difference of logits to the maximum add 4 u of their sizes.  With C = classes / 512 + 64 a log
probability is within u (C + 4 d + 4 |lse - m|) (d the distance to the maximum), p_j of the list
within u (C + 4 D) of itself: the argument D of its exponential is (the list's largest t - t) /
tau, of two roundings (3 u of itself), and |t| where t is a log probability.  From `stats` a q is within another 4 u (|z| / tau + |lse|).  A
bfloat16 gradient is rounded once more, 2^-8 of its value."""
import math

import pytest
import torch

import paper_2607_20548_amd as soap

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def reference(z, index, t, tau, tail):
    """loss, dlogits for dloss = 1, and the bounds of both, in float64."""
    rows, classes = z.shape
    z, t, index = z.double() / tau, t.double(), index.long()
    live = (index >= 0) & (index < classes)
    at = index.clamp(0, classes - 1)
    some = live.any(1)
    C = classes / 512 + 64
    most = z.amax(1, keepdim=True)
    most = torch.where(most.isinf(), 0.0, most)
    far_t = t.masked_fill(~live, 0.0).abs() if tail else \
        ((t.masked_fill(~live, -math.inf).amax(1, keepdim=True) - t) / tau).masked_fill(~live, 0.0).clamp_max(1e4)
    lse = torch.logsumexp(z, 1, keepdim=True)
    q = torch.where(z == -math.inf, 0.0, (z - lse).exp())
    if tail:
        logp = t.masked_fill(~live, -math.inf)
    else:
        logp = (t / tau).masked_fill(~live, -math.inf)
        logp = logp - torch.where(some[:, None], torch.logsumexp(logp, 1, keepdim=True), 0.0)
    p = torch.where(live, logp.exp(), 0.0)
    mass = p.sum(1)
    listed = torch.zeros(rows, classes, device=z.device, dtype=torch.int32).scatter_add_(1, at, live.int()) > 0
    rest = (1 - mass).clamp_min(0) * some if tail else torch.zeros_like(mass)
    lse_rest = torch.logsumexp(z.masked_fill(listed, -math.inf), 1, keepdim=True)
    rest = torch.where(lse_rest[:, 0] == -math.inf, 0.0, rest)
    logq = z.gather(1, at) - lse
    terms = torch.where(p > 0, p * (logp - logq), 0.0)
    d = most - z.gather(1, at)
    size = p * (C + 4 * torch.where(p > 0, d.abs() + logp.abs() + logq.abs(), 0.0) + 4 * (lse - most).abs()
                + torch.where(p > 0, (logp - logq).abs() * (C + 4 * far_t.nan_to_num()), 0.0))
    share = torch.where(rest > 0, lse_rest[:, 0] - lse[:, 0], 0.0)
    tailed = torch.where(rest > 0, rest * (rest.clamp_min(1e-300).log() - share), 0.0)
    # the rest is a difference of numbers near 1, and moves its term by its log's derivative
    rest_size = torch.where(rest > 0, rest * (C + 4 * share.abs() + 4 * (lse - most).abs()[:, 0])
                            + (C + 64) * (2 + (rest.clamp_min(1e-300).log() - share).abs()), 0.0)
    loss = tau ** 2 * (terms.sum(1) + tailed)
    loss_bound = tau ** 2 * U * (size.sum(1) + rest_size + C * terms.abs().sum(1))
    weight = (mass + rest)[:, None]
    qr = torch.where(listed | (z == -math.inf), 0.0, (z - lse_rest).exp()) * (rest > 0)[:, None]
    spread = C + 4 * (most - z).clamp_max(1e4) + 4 * (lse - most).abs()
    ps = torch.zeros_like(z).scatter_add_(1, at, p)
    pb = torch.zeros_like(z).scatter_add_(1, at, p * (C + 4 * far_t.nan_to_num(0, 0, 0)))
    dz = tau * (weight * q - rest[:, None] * qr - ps) * some[:, None]
    far = 4 * (z.abs().clamp_max(1e4) + lse.abs())
    bound = lambda extra: tau * U * ((q * weight + rest[:, None] * qr) * (spread + extra) + pb   # noqa: E731
                                     + ((C + 64) * qr if tail else 0))
    return loss, loss_bound, dz, bound(0), bound(far)


def within(got, want, bound, what):
    got = got.double()
    same = torch.isinf(want) & (got == want)
    bad = ~(((got - want).abs() <= bound) | same)
    assert not bad.any(), (what, int(bad.sum()), (got - want)[bad][:4].tolist(), bound[bad][:4].tolist())


def check(logits, index, teacher, tau=1.0, tail=False, dloss=None):
    rows, classes = logits.shape
    d = soap.Distillation(temperature=tau, tail=tail)
    if dloss is None:
        dloss = 0.5 + torch.rand(rows, device="cuda")
    want, loss_bound, dz, near, far = reference(logits, index, teacher, tau, tail)
    loss, stats = d.forward(logits, index, teacher)
    within(loss, want, loss_bound + 1e-30, "loss")
    both, dboth = d.forward_backward(logits, index, teacher, dloss)
    within(both, want, loss_bound + 1e-30, "loss of both")
    apart = d.backward(logits, index, teacher, stats, dloss)
    g = dloss.double()[:, None]
    step = 2.0 ** -8 if logits.dtype == torch.bfloat16 else 4 * U
    for got, bound, what in ((dboth, near, "dlogits of both"), (apart, far, "dlogits")):
        assert got.dtype == logits.dtype and got.shape == logits.shape
        within(got, g * dz, g.abs() * (bound * (1 + step) + step * dz.abs()) + 1e-36, what)
    return loss, dboth


def make(rows, classes, slots, dtype, seed, scale=3.0, tail=False, tau=1.0, t_dtype=torch.float32):
    z = scale * randn(seed, rows, classes)
    t = z + randn(seed + 1, rows, classes)
    k = min(slots, classes)
    top, index = t.topk(k, 1)
    if tail:
        top = top - torch.logsumexp(t, 1, keepdim=True)
    index = torch.nn.functional.pad(index.int(), (0, slots - k), value=-1)
    return z.to(dtype), index, torch.nn.functional.pad(top, (0, slots - k), value=math.nan).to(t_dtype)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,classes,slots", [
    (3, 1, 1), (2, 2, 3), (4, 7, 7), (5, 8, 2), (3, 100, 512), (600, 257, 5), (4, 4095, 64), (3, 4099, 17), (2, 8190, 1),
    (3, 8193, 33), (2, 16380, 100), (2, 32768, 16), (2, 50001, 100), (1, 65537, 256), (2, 131071, 64), (1, 150000, 512),
    (1, 262144, 64)])
def test_sizes(rows, classes, slots, dtype, tail):
    check(*make(rows, classes, slots, dtype, rows + classes, tail=tail), tail=tail)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("classes", [1023, 1024, 1025, 2048, 2056, 2560, 2561, 4095, 4096, 5120, 5121, 8192, 8200, 8201, 16384, 16392])
def test_many_rows(classes, dtype):
    """More rows than workgroups, which hold a row and fetch the next, on both sides of each of their
    widths."""
    check(*make(1500, classes, 12, dtype, classes), tail=False)
    check(*make(530, classes, 12, dtype, classes, tail=True), tail=True)


@pytest.mark.parametrize("tau", [0.05, 0.5, 2.0, 30.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_temperatures(dtype, tau):
    check(*make(4, 3001, 20, dtype, 5, t_dtype=torch.bfloat16), tau=tau)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_views(dtype, tail):
    """Rows at every alignment, in and out, lists cut from wider ones."""
    z, index, t = make(6, 1003, 9, dtype, 8, tail=tail)
    for off in range(9):
        wide = torch.full((6, 1003 + off + 1), 1e4, device="cuda", dtype=dtype)
        wide[:, off:off + 1003] = z
        iw, tw = torch.full((6, 12), 3, device="cuda", dtype=torch.int32), torch.full((6, 12), 9.0, device="cuda")
        iw[:, 1:10], tw[:, 1:10] = index, t
        check(wide[:, off:off + 1003], iw[:, 1:10], tw[:, 1:10], tail=tail)


@pytest.mark.parametrize("tail", [False, True])
def test_lists(tail):
    """Empty slots and lists, classes listed twice and many times, indices out of range, p of zero."""
    z, index, t = make(8, 500, 40, torch.float32, 3, tail=tail)
    index[0] = -1
    index[1, 1:] = -1
    index[2, 5:9] = index[2, 4]
    t[2, 4:9] -= math.log(5)
    index[3, ::2] = 500
    index[4, 7] = 2 ** 31 - 1
    index[5, 7] = -2 ** 31
    t[6, 3] = -math.inf
    index[7, :] = index[7, 0]
    t[7] -= math.log(40)
    t[0] = math.nan
    loss, dz = check(z, index, t, tail=tail)
    assert loss[0] == 0 and not dz[0].any()


@pytest.mark.parametrize("t_dtype", [torch.float32, torch.bfloat16])
def test_teacher_of_no_weight(t_dtype):
    """A list whose teacher has no logit above -inf weighs nothing, as an empty one: loss and gradient are
    zeros, in every call, and the other rows' as they are without it."""
    z, index, t = make(6, 700, 70, torch.float32, 13, t_dtype=t_dtype)
    clean = t.clone()
    t[1] = -math.inf
    t[3, :2], index[3, 2:] = -math.inf, -1
    t[4, 5] = -math.inf
    clean[4, 5] = -math.inf
    d = soap.Distillation(2.0)
    loss, stats = d.forward(z, index, t)
    both, dz = d.forward_backward(z, index, t)
    apart = d.backward(z, index, t, stats)
    want, dwant = d.forward_backward(z, index, clean)
    for r in (1, 3):
        assert loss[r] == 0 and both[r] == 0 and not dz[r].any() and not apart[r].any()
    for r in (0, 2, 4, 5):
        assert torch.equal(loss[r], want[r]) and torch.equal(both[r], want[r]) and torch.equal(dz[r], dwant[r])


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_logits(dtype, tail):
    """Classes at -inf and at the type's lowest value, all but the list, all but one."""
    z, index, t = make(6, 300, 6, dtype, 4, tail=tail)
    out = torch.ones(300, dtype=torch.bool, device="cuda")
    z[0, ~torch.isin(torch.arange(300, device="cuda"), index[0].long())] = -math.inf
    z[1, 100:200] = torch.finfo(dtype).min
    keep = index[2, :1].long()
    out[keep] = False
    z[2, out] = -math.inf
    index[2, 1:] = -1
    z[3, 50:] = -math.inf
    index[3] = torch.arange(6, device="cuda")
    z[4] = torch.finfo(dtype).min
    z[5] = 40000.0
    d = soap.Distillation(tail=tail)
    check(z[:4], index[:4], t[:4], tail=tail)
    # equal logits, however large: q is uniform, in the passes that see the logits
    loss, dz = d.forward_backward(z[4:], index[4:], t[4:])
    want, bound, g, near, _ = reference(torch.zeros_like(z[4:]), index[4:], t[4:], 1.0, tail)
    within(loss, want, 2 * bound, "loss")
    within(dz, g, 2 * near + 2.0 ** -7 * g.abs(), "dlogits")
    # p above zero on a class at -inf
    z[3, 2] = -math.inf
    assert d.forward(z, index, t)[0][3] == math.inf


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype,tau", [(torch.float32, 1.0), (torch.float32, 0.05), (torch.bfloat16, 1.0), (torch.bfloat16, 3.0)])
@pytest.mark.parametrize("rows,classes", [(6, 300), (520, 2500), (7, 70000)])
def test_gradient_from_stats_of_large_logits(rows, classes, dtype, tau, tail):
    """Rows whose log of the sums has no digits left of the sum: their gradient from forward's stats is as
    near to the formula as the single pass', which sees the logits (equal ones at the type's lowest value and
    elsewhere, and others at some distance from zero)."""
    z, index, t = make(rows, classes, 6, dtype, 4, tail=tail)
    z[0] = torch.finfo(dtype).min
    z[1] = 40000.0
    z[2] = (z[2].float() + 40000.0).to(dtype)
    z[3] = (4096.0 * z[3].float() - 1e6).to(dtype)
    z[4] = -1e30
    d = soap.Distillation(temperature=tau, tail=tail)
    dloss = 0.5 + torch.rand(rows, device="cuda")
    loss, stats = d.forward(z, index, t)
    moved = z.double() - z.double().amax(1, keepdim=True)
    want, loss_bound, dz, bound, _ = reference(moved, index, t, tau, tail)
    within(loss, want, loss_bound + 1e-30, "loss")
    both = d.forward_backward(z, index, t, dloss)[1]
    apart = d.backward(z, index, t, stats, dloss)
    g = dloss.double()[:, None]
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 4 * U
    for got, what in ((both, "dlogits of both"), (apart, "dlogits")):
        within(got, g * dz, g.abs() * (bound * (1 + step) + step * dz.abs()) + 1e-36, what)


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_from_logs(tail):
    """Stats of the two logs alone, as a caller's own forward pass has them."""
    z, index, t = make(40, 1001, 9, torch.float32, 17, tail=tail)
    d = soap.Distillation(temperature=0.7, tail=tail)
    _, stats = d.forward(z, index, t)
    *_, dz, _, far = reference(z, index, t, 0.7, tail)
    listed = torch.zeros(z.shape, device="cuda", dtype=torch.int32).scatter_add_(1, index.long(), torch.ones_like(index)) > 0
    logs = torch.logsumexp(z.double() / 0.7, 1), torch.logsumexp(z.double().masked_fill(listed, -math.inf) / 0.7, 1)
    logs = torch.stack([logs[0], logs[1] if tail else torch.zeros_like(logs[1])], 1)
    # a sum of C terms (as above), a log, and the logit added to it
    assert ((stats[:, :2] - logs).abs() <= (1001 / 512 + 72 + 4 * logs.abs()) * U).all()
    for given in (stats[:, :2].contiguous(), logs.float()):
        within(d.backward(z, index, t, given), dz, far * (1 + 4 * U) + 4 * U * dz.abs(), "dlogits")
    with pytest.raises(ValueError):
        d.backward(z, index, t, stats[:, :3].contiguous())
    with pytest.raises(ValueError):
        d.backward(z, index, t, stats[:, :2])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rest_of_lowest_logits(dtype):
    """With a tail, logits at the type's lowest value and a temperature under which their log of sums
    passes fp32's range: the classes outside the list still take the rest."""
    z, index, t = make(3, 300, 6, dtype, 4, tail=True)
    z[:] = torch.finfo(dtype).min
    d = soap.Distillation(temperature=0.25, tail=True)
    want, loss_bound, dz, bound, _ = reference(torch.zeros_like(z), index, t, 0.25, True)
    loss, both = d.forward_backward(z, index, t)
    within(loss, want, loss_bound, "loss of both")
    within(d.forward(z, index, t)[0], want, loss_bound, "loss")
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 4 * U
    within(both, dz, bound * (1 + step) + step * dz.abs(), "dlogits")


def test_not_numbers():
    """NaN and +inf stay in their row; rows without a list, and of dloss 0, are zeros all the same."""
    z, index, t = make(6, 3000, 5, torch.float32, 6)
    clean = z.clone()
    z[1, 7], z[2, 2999], z[3, 0], z[4] = math.nan, math.inf, math.nan, math.nan
    index[3] = -1
    dloss = torch.ones(6, device="cuda")
    dloss[4] = 0
    d = soap.Distillation()
    loss, dz = d.forward_backward(z, index, t, dloss)
    _, stats = d.forward(z, index, t)
    apart = d.backward(z, index, t, stats, dloss)
    want, dwant = d.forward_backward(clean, index, t, dloss)
    for g in (dz, apart):
        assert g[1].isnan().all() and g[2].isnan().any() and not g[3].any() and not g[4].any()
    for r in (0, 5):
        assert torch.equal(loss[r], want[r]) and torch.equal(dz[r], dwant[r])
    assert loss[1].isnan() and loss[2].isnan() and loss[3] == 0


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_logit(dtype, tail):
    """Rows whose logits are all -inf: NaN, but zeros for an empty list and a dloss of 0; the other rows'
    bits are as without them."""
    z, index, t = make(6, 999, 5, dtype, 19, tail=tail)
    clean, dloss = z.clone(), torch.ones(6, device="cuda")
    z[[1, 3, 4]] = -math.inf
    index[3] = -1
    dloss[4] = 0
    d = soap.Distillation(tail=tail)
    loss, dz = d.forward_backward(z, index, t, dloss)
    alone, stats = d.forward(z, index, t)
    want, dwant = d.forward_backward(clean, index, t, dloss)
    assert loss[1].isnan() and loss[4].isnan() and loss[3] == 0 and torch.equal(loss.nan_to_num(9), alone.nan_to_num(9))
    for g in (dz, d.backward(z, index, t, stats, dloss)):
        listed = torch.zeros(999, dtype=torch.bool, device="cuda")
        listed[index[1].long()] = True
        assert g[1, listed].isnan().all() and (not g[1, ~listed].any() if tail else g[1].isnan().all())
        assert not g[3].any() and not g[4].any()
    for r in (0, 2, 5):
        assert torch.equal(loss[r], want[r]) and torch.equal(dz[r], dwant[r])


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_against_differences(tail):
    """<gradient, v> against the kernel's own losses half a step on either side: h^2 of the third
    derivative (below 8 h^2 tau^-1 for |v| <= 1) and the losses' rounding over h."""
    tau = 1.0 if tail else 2.0
    z, index, t = make(3, 64, 7, torch.float32, 9, tail=tail)
    v = 2 * torch.rand(3, 64, device="cuda") - 1
    d, h = soap.Distillation(temperature=tau, tail=tail), 2.0 ** -6
    _, dz = d.forward_backward(z, index, t)
    hi, lo = (d.forward(z + s * h * v, index, t)[0].double() for s in (1, -1))
    want, got = (hi - lo) / (2 * h), (dz.double() * v).sum(1)
    _, bound, *_ = reference(z, index, t, tau, tail)
    assert ((got - want).abs() <= 8 * h * h / tau + 2 * bound / h).all()


def test_cross_entropy_to_labels():
    """A list of one slot is the cross entropy to a label."""
    z = 2 * randn(1, 50, 1000)
    label = torch.randint(0, 1000, (50, 1), device="cuda", dtype=torch.int32)
    loss, dz = soap.Distillation().forward_backward(z, label, torch.zeros(50, 1, device="cuda"))
    want = torch.logsumexp(z.double(), 1) - z.double().gather(1, label.long())[:, 0]
    assert ((loss.double() - want).abs() <= 64 * U * (1 + want + 16)).all()
    assert (dz.sum(1).abs() <= 1e-5).all()


def test_rows_past_32_bits():
    """Rows whose offset passes 2^31 elements: 20 000 of 131 072 bfloat16 logits."""
    rows, classes = 20000, 131072
    z = torch.zeros(rows, classes, device="cuda", dtype=torch.bfloat16)
    z[:, 5] = 3.0
    z[-1] = randn(1, classes)
    index = torch.full((rows, 2), 5, device="cuda", dtype=torch.int32)
    index[:, 1] = -1
    index[-1, 1] = 77
    t = torch.zeros(rows, 2, device="cuda")
    d = soap.Distillation()
    loss, dz = d.forward_backward(z, index, t)
    want, bound, g, near, _ = reference(z[-2:], index[-2:], t[-2:], 1.0, False)
    within(loss[-2:], want, bound, "loss")
    within(dz[-2:], g, near + 2.0 ** -8 * g.abs() + 1e-36, "dlogits")
    assert (loss[:-1] == loss[0]).all() and torch.equal(dz[0], dz[-2]) and torch.equal(dz[12345], dz[0])


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rows,classes,dtype", [
    (27000, 1000, torch.float32), (27000, 2000, torch.bfloat16), (9000, 3000, torch.float32), (9000, 6000, torch.bfloat16),
    (1100, 24000, torch.float32), (1100, 48000, torch.bfloat16), (600, 50001, torch.float32), (600, 100001, torch.bfloat16),
    (300, 100001, torch.float32), (300, 200001, torch.bfloat16), (520, 33000, torch.float32), (520, 66000, torch.bfloat16)])
def test_loss_and_gradient_apart(rows, classes, dtype, tail):
    """Loss and gradient by themselves of more than the caches hold, for each number of threads, and many
    rows of the most threads."""
    check(*make(rows, classes, 9, dtype, classes, tail=tail), tail=tail)


def test_apart_past_32_bits():
    """Loss and gradient by themselves of rows past 2^31 elements, with and without a tail: the last rows as they
    are alone, to the rounding of their sums in another number of threads."""
    rows, classes, last = 20000, 131072, 3
    z = torch.zeros(rows, classes, device="cuda", dtype=torch.bfloat16)
    z[-last:] = randn(1, last, classes)
    index = torch.full((rows, 2), 5, device="cuda", dtype=torch.int32)
    index[:, 1] = 77
    t = torch.full((rows, 2), -2.0, device="cuda")
    for tail in (False, True):
        d = soap.Distillation(tail=tail)
        loss, stats = d.forward(z, index, t)
        dz = d.backward(z, index, t, stats)
        want, bound, g, near, _ = reference(z[-last:], index[-last:], t[-last:], 1.0, tail)
        within(loss[-last:], want, bound, "loss")
        within(dz[-last:], g, near + 2.0 ** -8 * (g.abs() + near) + 1e-36, "dlogits")
        assert (loss[:-last] == loss[0]).all() and torch.equal(dz[0], dz[-last - 1]) and torch.equal(dz[16384], dz[0])
        del dz


def test_most_rows():
    """As many rows as a call takes, in each of the three: the last ones as they are alone."""
    rows, last = 1 << 24, 1000
    z = (torch.arange(rows * 3, device="cuda") % 1009 / 200.0).view(rows, 3).bfloat16()
    index = (torch.arange(rows, device="cuda", dtype=torch.int32) % 3)[:, None]
    t = torch.zeros(rows, 1, device="cuda")
    d = soap.Distillation()
    loss, stats = d.forward(z, index, t)
    dz = d.backward(z, index, t, stats)
    both, dz_both = d.forward_backward(z, index, t)
    want, want_stats = d.forward(z[-last:], index[-last:], t[-last:])
    assert torch.equal(loss[-last:], want) and torch.equal(stats[-last:], want_stats)
    assert torch.equal(dz[-last:], d.backward(z[-last:], index[-last:], t[-last:], want_stats))
    want, want_dz = d.forward_backward(z[-last:], index[-last:], t[-last:])
    assert torch.equal(both[-last:], want) and torch.equal(dz_both[-last:], want_dz)


def test_no_rows():
    d = soap.Distillation()
    z, index, t = torch.empty(0, 10, device="cuda"), torch.empty(0, 2, device="cuda", dtype=torch.int32), torch.empty(0, 2, device="cuda")
    loss, dz = d.forward_backward(z, index, t)
    assert loss.shape == (0,) and dz.shape == (0, 10)
    loss, stats = d.forward(z, index, t)
    assert d.backward(z, index, t, stats).shape == (0, 10)


@pytest.mark.parametrize("classes", [900, 40000])
def test_stream_graph_and_bits(classes):
    z, index, t = make(40, classes, 30, torch.bfloat16, 11, tail=True)
    d = soap.Distillation(tail=True)
    dloss = torch.rand(40, device="cuda")

    def run(**kw):
        loss, stats = d.forward(z, index, t, **kw)
        return (loss, stats, d.backward(z, index, t, stats, dloss, **kw), *d.forward_backward(z, index, t, dloss, **kw))

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
        z.copy_(3 * randn(30 + i, 40, classes))
        graph.replay()
        want = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), i
