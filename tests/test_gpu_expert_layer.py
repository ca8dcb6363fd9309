"""The layer of experts (examples/expert_layer.py): all operators together.

Its gradients are compared with those of the same layer in float64 without any
rounding to 4 bits.  A value in MXFP4 is off by at most a quarter of itself and, over
values spread evenly between levels, by about 0.12 of it (rms); a product of two such
operands by sqrt(2) 0.12 = 0.17 and a gradient that went through two of them by 0.24,
so that the angle to the exact gradient has a cosine of at least 0.97; the bound is
0.95."""
import os
import sys

import pytest
import torch

import paper_2607_20548_amd as soap

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
import expert_layer  # noqa: E402

pytestmark = pytest.mark.gpu


def cosine(a, b):
    a, b = a.double().reshape(-1), b.double().reshape(-1)
    return (a @ b / (a.norm() * b.norm())).item()


@pytest.mark.parametrize("tokens,experts,k,m,n", [(300, 8, 2, 128, 96), (77, 12, 3, 160, 64)])
def test_gradients(tokens, experts, k, m, n):
    layer = expert_layer.ExpertLayer(experts, k, m, n, seed=3, balance=0.05)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(tokens, m, generator=g, device="cuda").bfloat16()
    layer.weight += 0.2 * torch.randn(m, generator=g, device="cuda")
    layer.bias += 0.1 * torch.randn(m, generator=g, device="cuda")
    y = layer.forward(x)
    dy = torch.randn(tokens, n, generator=g, device="cuda")
    got = layer.backward(dy)
    r = layer.kept[7]
    p = {"x": x, "weight": layer.weight, "bias": layer.bias, "route": layer.route, "bank": layer.bank}
    p = {name: t.double().requires_grad_(True) for name, t in p.items()}
    var, mean = torch.var_mean(p["x"], dim=1, correction=0, keepdim=True)
    h = (p["x"] - mean) * torch.rsqrt(var + 1e-5) * p["weight"] + p["bias"]
    prob = torch.softmax(h @ p["route"], 1)
    index = r.index.long()
    gate = prob.gather(1, index)
    gate = gate / gate.sum(1, keepdim=True)
    out = torch.einsum("tm,tkmn->tkn", h, p["bank"][index])
    ref = (out * gate[..., None]).sum(1)
    counts = r.counts.double()
    balance = 0.05 * experts * (counts[:-1] / counts[:-1].sum() * prob.mean(0)).sum()
    ((ref * dy.double()).sum() + balance).backward()
    assert cosine(y, ref) >= 0.95
    for name, t in p.items():
        assert got[name].shape == t.shape
        assert cosine(got[name], t.grad) >= 0.95, name
    idle = (counts[:-1] == 0).nonzero().view(-1)
    assert (got["bank"][idle] == 0).all()


@pytest.mark.parametrize("optimizer", ["muon", "soap"])
def test_it_learns_and_repeats(optimizer):
    run = lambda: expert_layer.train(300, 8, 2, 128, 64, 8, optimizer=optimizer, lr=0.1)  # noqa: E731
    losses = run()
    assert losses[-1] < 0.9 * losses[0] and all(b < a for a, b in zip(losses, losses[1:3]))
    assert losses == run()


def test_a_bank_of_idle_experts():
    """More experts than rows: most groups are empty."""
    layer = expert_layer.ExpertLayer(64, 2, 64, 32, seed=5)
    x = torch.randn(3, 64, device="cuda").bfloat16()
    y = layer.forward(x)
    got = layer.backward(torch.ones_like(y))
    busy = torch.zeros(64, dtype=torch.bool, device="cuda")
    busy[layer.kept[7].index.view(-1).long()] = True
    assert torch.equal(got["bank"].abs().sum((1, 2)) > 0, busy)
    assert not y.isnan().any() and not got["x"].isnan().any()
