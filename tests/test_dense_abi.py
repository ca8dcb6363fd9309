"""Argument checks of the dense layer's entry points (no GPU): every refusal comes before
anything is enqueued, with its documented status and a message; only fake pointers are passed, and
only to calls that must fail.  The classes refuse host tensors and wrong shapes themselves."""
import random

import pytest
import torch

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


def head_fwd(L, **o):
    a = dict(tokens=8, q_heads=4, k_heads=2, dim=32, rotary=32, dtype=soap.SOAP_BF16, flags=0, q=P(0), q_token=128,
             q_head=32, k=P(1), k_token=64, k_head=32, q_weight=P(2), k_weight=P(3), eps=1e-6, positions=P(4),
             frequencies=P(5), q_out=P(6), q_out_token=128, q_out_head=32, k_out=P(7), k_out_token=64, k_out_head=32)
    a.update(o)
    return L.soap_head_norm_forward(*a.values(), None)


HEAD_REFUSALS = [
    (dict(tokens=-1), soap.SOAP_ERR_SHAPE),
    (dict(tokens=soap.SOAP_MAX_ROWS + 1), soap.SOAP_ERR_SHAPE),
    (dict(q_heads=-1), soap.SOAP_ERR_SHAPE),
    (dict(k_heads=soap.SOAP_HEAD_MAX_HEADS + 1), soap.SOAP_ERR_SHAPE),
    (dict(dim=0), soap.SOAP_ERR_SHAPE),
    (dict(dim=33), soap.SOAP_ERR_SHAPE),
    (dict(dim=soap.SOAP_HEAD_MAX_DIM + 2), soap.SOAP_ERR_SHAPE),
    (dict(rotary=34), soap.SOAP_ERR_SHAPE),
    (dict(rotary=7), soap.SOAP_ERR_SHAPE),
    (dict(rotary=-2), soap.SOAP_ERR_SHAPE),
    (dict(dtype=2), soap.SOAP_ERR_HPARAM),
    (dict(flags=2), soap.SOAP_ERR_HPARAM),
    (dict(eps=0.0), soap.SOAP_ERR_HPARAM),
    (dict(eps=float("inf")), soap.SOAP_ERR_HPARAM),
    (dict(q=None), soap.SOAP_ERR_NULL),
    (dict(k=None), soap.SOAP_ERR_NULL),
    (dict(frequencies=None), soap.SOAP_ERR_NULL),
    (dict(frequencies=P(5, 4)), soap.SOAP_ERR_ALIGN),
    (dict(q=P(0, 1)), soap.SOAP_ERR_ALIGN),
    (dict(positions=P(4, 2)), soap.SOAP_ERR_ALIGN),
    (dict(q_token=-1), soap.SOAP_ERR_SHAPE),
    (dict(k_head=1 << 31), soap.SOAP_ERR_SHAPE),
]


@pytest.mark.parametrize("over,code", HEAD_REFUSALS + [
    (dict(q_out=None), soap.SOAP_ERR_NULL),
    (dict(q_out_head=31), soap.SOAP_ERR_ALIAS),           # heads over each other
    (dict(q_out_token=127), soap.SOAP_ERR_ALIAS),         # tokens over each other
    (dict(q_out_token=0), soap.SOAP_ERR_ALIAS),
    (dict(q_out=P(0)), soap.SOAP_ERR_ALIAS),              # in place
    (dict(q_out=P(1)), soap.SOAP_ERR_ALIAS),              # over the keys
    (dict(k_out=P(6, 2 * 127)), soap.SOAP_ERR_ALIAS),     # over the queries' outputs
    (dict(k_out=P(4)), soap.SOAP_ERR_ALIAS),
])
def test_head_norm_forward_refuses(L, over, code):
    assert head_fwd(L, **over) == code
    assert soap.soap_last_error() != ""


def head_bwd(L, **o):
    a = dict(tokens=8, q_heads=4, k_heads=2, dim=32, rotary=32, dtype=soap.SOAP_F32, flags=1, dq_out=P(0), dq_out_token=128,
             dq_out_head=32, dk_out=P(1), dk_out_token=64, dk_out_head=32, q=P(2), q_token=128, q_head=32, k=P(3),
             k_token=64, k_head=32, q_weight=P(4), k_weight=P(5), eps=1e-6, positions=P(6), frequencies=P(7), dq=P(8),
             dq_token=128, dq_head=32, dk=P(9), dk_token=64, dk_head=32, dq_weight=P(10), dk_weight=P(11), ws=P(12),
             wsb=soap.soap_head_norm_workspace_bytes(8, 32))
    a.update(o)
    return L.soap_head_norm_backward(*a.values(), None)


@pytest.mark.parametrize("over,code", [(o, c) for o, c in HEAD_REFUSALS if o != dict(flags=2)] + [
    (dict(dq_out=None), soap.SOAP_ERR_NULL),
    (dict(ws=None), soap.SOAP_ERR_NULL),
    (dict(wsb=15), soap.SOAP_ERR_WORKSPACE),
    (dict(ws=P(12, 8)), soap.SOAP_ERR_ALIGN),
    (dict(dq=P(2)), soap.SOAP_ERR_ALIAS),
    (dict(dq=P(1)), soap.SOAP_ERR_ALIAS),
    (dict(dk=P(8)), soap.SOAP_ERR_ALIAS),
    (dict(dk=P(8, 4 * 96), dk_token=128, dq_token=128), soap.SOAP_ERR_ALIAS),   # one head into the next token's
    (dict(dq_weight=P(4)), soap.SOAP_ERR_ALIAS),
    (dict(dk_weight=P(10)), soap.SOAP_ERR_ALIAS),
    (dict(dq_head=16), soap.SOAP_ERR_ALIAS),
])
def test_head_norm_backward_refuses(L, over, code):
    assert head_bwd(L, **over) == code


def interleaved(at, ahead, bt, bhead, at_b, tokens=8, qh=4, kh=2):
    """Strides for dq and dk in one buffer, dk `at_b` floats behind it."""
    return dict(tokens=tokens, q_heads=qh, k_heads=kh, dq=P(8), dq_token=at, dq_head=ahead, dk=P(8, 4 * at_b),
                dk_token=bt, dk_head=bhead, q_token=qh * 32, dq_out_token=qh * 32, k_token=kh * 32, dk_out_token=kh * 32)


@pytest.mark.parametrize("over,code", [
    # heads of both in turn in a token's row, and in heads in front of tokens
    (interleaved(256, 64, 256, 64, 32), soap.SOAP_ERR_WORKSPACE),
    (interleaved(256, 64, 256, 64, 32 + 2 * 64), soap.SOAP_ERR_WORKSPACE),
    (interleaved(64, 512, 64, 512, 32), soap.SOAP_ERR_WORKSPACE),
    (interleaved(32, 512, 32, 512, 256), soap.SOAP_ERR_WORKSPACE),
    # one head between the other side's
    (interleaved(256, 64, 256, 7, 32, kh=1), soap.SOAP_ERR_WORKSPACE),
    (interleaved(256, 9, 256, 64, 32, qh=1), soap.SOAP_ERR_WORKSPACE),
    # one token: its strides say nothing
    (interleaved(256, 64, 99, 64, 32, tokens=1), soap.SOAP_ERR_WORKSPACE),
    # a value over another's
    (interleaved(256, 64, 256, 64, 31), soap.SOAP_ERR_ALIAS),
    (interleaved(256, 64, 256, 64, 33), soap.SOAP_ERR_ALIAS),
    (interleaved(64, 512, 64, 512, 33), soap.SOAP_ERR_ALIAS),
    (interleaved(32, 512, 32, 512, 255), soap.SOAP_ERR_ALIAS),
    (interleaved(32, 512, 32, 512, 257), soap.SOAP_ERR_ALIAS),
    (interleaved(256, 64, 256, 7, 33, kh=1), soap.SOAP_ERR_ALIAS),
    # in turn in the first token, not in the next ones
    (interleaved(256, 64, 288, 64, 32), soap.SOAP_ERR_ALIAS),
    # the last head of a token on the next token's first
    (interleaved(256, 64, 256, 64, 32 + 192), soap.SOAP_ERR_WORKSPACE),
    (interleaved(224, 64, 224, 64, 32 + 192), soap.SOAP_ERR_ALIAS),
    (interleaved(256, 64, 256, 64, 32 + 193), soap.SOAP_ERR_ALIAS),
])
def test_heads_in_turn(L, over, code):
    """Outputs between those of the other side are taken, as far as the workspace, which is too small."""
    assert head_bwd(L, wsb=15, **over) == code


def test_heads_in_turn_against_all_pairs(L):
    """Layouts of equal strides at random against every pair of heads."""
    rng, seen = random.Random(5), set()
    for _ in range(3000):
        tokens, qh, kh = rng.randint(1, 4), rng.randint(1, 3), rng.randint(1, 3)
        head, token = rng.choice([(16, 16 * rng.randint(4, 9)), (16 * rng.randint(1, 3), 128), (16 * rng.randint(4, 12), 16 * rng.randint(1, 4))])
        d = rng.choice([rng.randint(0, 700), 8 * rng.randint(0, 80)])
        a = dict(interleaved(token, head, token, head, d, tokens, qh, kh), dim=8, rotary=8, q_head=8, k_head=8,
                 dq_out_head=8, dk_out_head=8)
        rows = lambda h, o: [o + i * token + j * head for i in range(tokens) for j in range(h)]  # noqa: E731
        q, k = rows(qh, 0), rows(kh, d)
        apart = lambda u, v: all(abs(x - y) >= 8 for x in u for y in v)  # noqa: E731
        # a side's own heads: of a token, or tokens of a head, one behind the other
        nested = lambda h: token >= (h - 1) * head + 8 or tokens == 1 or head >= (tokens - 1) * token + 8 or h == 1  # noqa: E731
        if nested(qh) and nested(kh):
            code = head_bwd(L, wsb=15, **a)
            assert code == (soap.SOAP_ERR_WORKSPACE if apart(q, k) else soap.SOAP_ERR_ALIAS), (a, apart(q, k))
            seen.add(code)
    assert len(seen) == 2


def gated_fwd(L, **o):
    a = dict(tokens=8, m=64, n=72, p=80, act=soap.SOAP_ACT_SILU, x=P(0), ldx=64, wg=P(1), wu=P(2), wd=P(3), gate=P(4),
             up=P(5), y=P(6), ldy=80, ws=P(7), wsb=soap.soap_gated_workspace_bytes(8, 64, 72, 80, False))
    a.update(o)
    return L.soap_gated_forward(*a.values(), None)


GATED_REFUSALS = [
    (dict(tokens=-1), soap.SOAP_ERR_SHAPE),
    (dict(m=60), soap.SOAP_ERR_SHAPE),
    (dict(n=0), soap.SOAP_ERR_SHAPE),
    (dict(n=soap.SOAP_GATED_MAX_HIDDEN + 8), soap.SOAP_ERR_SHAPE),
    (dict(p=soap.SOAP_MAX_DIM + 8), soap.SOAP_ERR_SHAPE),
    (dict(p=84), soap.SOAP_ERR_SHAPE),
    (dict(act=2), soap.SOAP_ERR_HPARAM),
    (dict(ldx=56), soap.SOAP_ERR_SHAPE),
    (dict(ldx=68), soap.SOAP_ERR_SHAPE),
    (dict(ldx=soap.SOAP_GATED_MAX_LD + 8), soap.SOAP_ERR_SHAPE),
    (dict(x=None), soap.SOAP_ERR_NULL),
    (dict(wd=None), soap.SOAP_ERR_NULL),
    (dict(x=P(0, 8)), soap.SOAP_ERR_ALIGN),
    (dict(wu=P(2, 2)), soap.SOAP_ERR_ALIGN),
    (dict(wsb=100), soap.SOAP_ERR_WORKSPACE),
    (dict(ws=None), soap.SOAP_ERR_NULL),
]


@pytest.mark.parametrize("over,code", GATED_REFUSALS + [
    (dict(gate=None), soap.SOAP_ERR_NULL),
    (dict(ldy=72), soap.SOAP_ERR_SHAPE),
    (dict(y=None), soap.SOAP_ERR_NULL),
    (dict(y=P(0)), soap.SOAP_ERR_ALIAS),
    (dict(up=P(4)), soap.SOAP_ERR_ALIAS),
    (dict(ws=P(1)), soap.SOAP_ERR_ALIAS),
])
def test_gated_forward_refuses(L, over, code):
    assert gated_fwd(L, **over) == code


def gated_bwd(L, **o):
    a = dict(tokens=8, m=64, n=72, p=80, act=soap.SOAP_ACT_GELU, dy=P(0), lddy=80, x=P(1), ldx=64, wg=P(2), wu=P(3),
             wd=P(4), gate=P(5), up=P(6), dx=P(7), lddx=64, dtype=soap.SOAP_F32, dwg=P(8), dwu=P(9), dwd=P(10), ws=P(11),
             wsb=soap.soap_gated_workspace_bytes(8, 64, 72, 80, True))
    a.update(o)
    return L.soap_gated_backward(*a.values(), None)


@pytest.mark.parametrize("over,code", [(o, c) for o, c in GATED_REFUSALS if "wu" not in o] + [
    (dict(lddy=88 - 4), soap.SOAP_ERR_SHAPE),
    (dict(lddx=56), soap.SOAP_ERR_SHAPE),
    (dict(dtype=3), soap.SOAP_ERR_HPARAM),
    (dict(gate=None), soap.SOAP_ERR_NULL),
    (dict(dwg=P(8, 4)), soap.SOAP_ERR_ALIGN),
    (dict(dx=P(1)), soap.SOAP_ERR_ALIAS),
    (dict(dwu=P(8)), soap.SOAP_ERR_ALIAS),
    (dict(dwd=P(4)), soap.SOAP_ERR_ALIAS),
])
def test_gated_backward_refuses(L, over, code):
    assert gated_bwd(L, **over) == code


def distill(L, which, **o):
    a = dict(rows=4, classes=100, slots=3, dtype=soap.SOAP_BF16, logits=P(0), ld=100, index=P(1), ldi=3,
             teacher_dtype=soap.SOAP_F32, teacher=P(2), ldt=3, flags=0, temperature=1.0)
    more = dict(forward=dict(loss=P(3), stats=P(4)), backward=dict(stats=P(4), dloss=P(5), dlogits=P(6), ldd=100),
                forward_backward=dict(dloss=P(5), loss=P(3), stats=P(4), dlogits=P(6), ldd=100))[which]
    a.update(more)
    a.update({k: v for k, v in o.items()})
    return getattr(L, "soap_distill_" + which)(*a.values(), None)


@pytest.mark.parametrize("which", ["forward", "backward", "forward_backward"])
@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), soap.SOAP_ERR_SHAPE),
    (dict(classes=0), soap.SOAP_ERR_SHAPE),
    (dict(classes=soap.SOAP_DISTILL_MAX_CLASSES + 1, ld=1 << 20), soap.SOAP_ERR_SHAPE),
    (dict(slots=0), soap.SOAP_ERR_SHAPE),
    (dict(slots=soap.SOAP_DISTILL_MAX_SLOTS + 1, ldi=1024, ldt=1024), soap.SOAP_ERR_SHAPE),
    (dict(dtype=2), soap.SOAP_ERR_HPARAM),
    (dict(teacher_dtype=-1), soap.SOAP_ERR_HPARAM),
    (dict(ld=99), soap.SOAP_ERR_SHAPE),
    (dict(ldi=2), soap.SOAP_ERR_SHAPE),
    (dict(ldt=2), soap.SOAP_ERR_SHAPE),
    (dict(flags=2), soap.SOAP_ERR_HPARAM),
    (dict(temperature=0.0), soap.SOAP_ERR_HPARAM),
    (dict(temperature=1000.0), soap.SOAP_ERR_HPARAM),
    (dict(temperature=float("nan")), soap.SOAP_ERR_HPARAM),
    (dict(logits=None), soap.SOAP_ERR_NULL),
    (dict(index=None), soap.SOAP_ERR_NULL),
    (dict(teacher=None), soap.SOAP_ERR_NULL),
    (dict(logits=P(0, 1)), soap.SOAP_ERR_ALIGN),
    (dict(index=P(1, 2)), soap.SOAP_ERR_ALIGN),
])
def test_distill_refuses(L, which, over, code):
    assert distill(L, which, **over) == code


@pytest.mark.parametrize("which,over,code", [
    ("forward", dict(loss=None), soap.SOAP_ERR_NULL),
    ("forward", dict(loss=P(1)), soap.SOAP_ERR_ALIAS),
    ("forward", dict(stats=P(3, 8)), soap.SOAP_ERR_ALIAS),
    ("backward", dict(stats=None), soap.SOAP_ERR_NULL),
    ("backward", dict(dlogits=None), soap.SOAP_ERR_NULL),
    ("backward", dict(ldd=99), soap.SOAP_ERR_SHAPE),
    ("backward", dict(dlogits=P(0)), soap.SOAP_ERR_ALIAS),
    ("forward_backward", dict(loss=None), soap.SOAP_ERR_NULL),
    ("forward_backward", dict(dlogits=None), soap.SOAP_ERR_NULL),
    ("forward_backward", dict(dlogits=P(5)), soap.SOAP_ERR_ALIAS),
])
def test_distill_outputs_refused(L, which, over, code):
    assert distill(L, which, **over) == code


@pytest.mark.parametrize("which", ["forward", "forward_backward"])
def test_distill_sums_take_six_floats(L, which):
    """A row of stats: two floats, or six with the sums; the loss lies behind four rows of two."""
    assert distill(L, which, stats=P(3), loss=P(3, 32), flags=soap.SOAP_DISTILL_SUMS) == soap.SOAP_ERR_ALIAS
    assert distill(L, which, flags=8) == soap.SOAP_ERR_HPARAM


def test_workspace_sizes(L):
    """Zero for sizes that are refused, and never less for a larger call."""
    assert soap.soap_head_norm_workspace_bytes(4, 1) == 0 and soap.soap_head_norm_workspace_bytes(-1, 64) == 0
    assert soap.soap_gated_workspace_bytes(4, 60, 64, 64, True) == 0
    grown = [soap.soap_head_norm_workspace_bytes(t, d) for t in (1, 100, 10000) for d in (64, 128)]
    assert grown[0] <= grown[1] and grown[0] <= grown[2] <= grown[4]
    for back in (False, True):
        for size in (dict(m=512), dict(n=1024), dict(p=512)):
            last = 0
            for t in (0, 1, 15, 16, 17, 100, 129, 300, 600, 1000, 2000, 5000, 20000):
                args = dict(m=256, n=512, p=256)
                now = soap.soap_gated_workspace_bytes(t, *args.values(), back)
                assert now >= last
                last = now
                args.update(size)
                assert soap.soap_gated_workspace_bytes(t, *args.values(), back) >= now


def test_classes_refuse():
    host = torch.zeros(4, 2, 32)
    with pytest.raises(ValueError):
        soap.HeadNorm(31, frequencies=torch.zeros(0, dtype=torch.float64))
    with pytest.raises(ValueError):
        soap.HeadNorm(32, rotary=40)
    with pytest.raises(ValueError):
        soap.HeadNorm(32, torch.ones(32))
    norm = soap.HeadNorm(32, rotary=0)
    for call in (lambda: norm.forward(host), lambda: norm.forward(None), lambda: norm.forward(None, host)):
        with pytest.raises(ValueError):
            call()
    w = torch.zeros(8, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        soap.GatedFeedForward(w, w, w)
    with pytest.raises(ValueError):
        soap.GatedFeedForward(w, w, w, activation="relu")
    for t in (0.0, -1.0, 1e9, float("nan")):
        with pytest.raises(ValueError):
            soap.Distillation(temperature=t)
    with pytest.raises(ValueError):
        soap.Distillation().forward(torch.zeros(2, 8), torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1))
