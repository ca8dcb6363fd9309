"""The operators of the layer around an expert bank, as timed cases: layer norm
forward and backward, the router with its balance loss, counts and dispatch
plan, and products in microscaled 4-bit floating point (MXFP4), dense and
grouped by the router's counts.

``listed()`` gives the cases, ``draw(rng)`` one more of the same ranges,
``prepare`` what a program holds before a call, ``run`` one call (the plain
form in 32-bit torch, or the package's kernels where ``own`` is true),
``exact`` its outputs from the definition in 64 bits and ``work`` the bytes and
flops a call cannot do without.

MXFP4: blocks of 32 values along the summed axis share the power of two
2^e, e = floor(log2 max|x|) - 2, and hold x / 2^e on {0, 0.5, 1, 1.5, 2, 3, 4,
6} (nearest, ties to even, saturated).  Packed rows hold two values a byte
(the lower half first) and a byte e + 127 per block, padded to 256 values.
"""
import math

import torch

own = False

EPS = 1e-5
BALANCE = 0.01
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def listed():
    return [
        # the norm of one token, as a served model calls it: latency
        {"name": "norm_1x2048", "kind": "norm", "rows": 1, "cols": 2048, "dtype": "bf16", "pad": 0},
        # the norm in front of a 4096-wide layer, a batch of 4 sequences of 4096 tokens
        {"name": "norm_16384x4096", "kind": "norm", "rows": 16384, "cols": 4096, "dtype": "bf16", "pad": 0},
        # its backward pass, with the reduction of the weight's gradient over all tokens
        {"name": "norm_grad_16384x4096", "kind": "norm_grad", "rows": 16384, "cols": 4096,
         "dtype": "bf16", "pad": 0},
        # odd sizes, rows cut out of a wider tensor
        {"name": "norm_grad_1101x2303", "kind": "norm_grad", "rows": 1101, "cols": 2303, "dtype": "fp32",
         "pad": 5},
        # routing of a few tokens: latency
        {"name": "route_8x64", "kind": "route", "tokens": 8, "experts": 64, "top_k": 8, "dtype": "fp32",
         "masked": 0.0, "renorm": True},
        # routing of a training batch, some of its tokens padding
        {"name": "route_32768x128", "kind": "route", "tokens": 32768, "experts": 128, "top_k": 8,
         "dtype": "bf16", "masked": 0.05, "renorm": True},
        # the gradient of gates and balance loss on the same batch
        {"name": "route_grad_32768x128", "kind": "route_grad", "tokens": 32768, "experts": 128, "top_k": 8,
         "dtype": "fp32", "masked": 0.05, "renorm": False},
        # the expert bank after an optimizer step: its 4-bit values for the forward
        # product and for the input gradient's, one pass over the weights
        {"name": "mx4_bank_64x2048x768", "kind": "mx4_bank", "batch": 64, "m": 2048, "n": 768},
        # the MLP up-projection of a training batch and of a few tokens
        {"name": "mx4_linear_8192x4096x14336", "kind": "mx4_linear", "tokens": 8192, "m": 4096, "n": 14336},
        {"name": "mx4_linear_16x4096x14336", "kind": "mx4_linear", "tokens": 16, "m": 4096, "n": 14336},
        # the bank's forward product on routed tokens, and its weight gradient
        {"name": "mx4_experts_64x2048x768", "kind": "mx4_experts", "experts": 64, "tokens": 4096, "top_k": 8,
         "m": 2048, "n": 768},
        {"name": "mx4_experts_grad_64x2048x768", "kind": "mx4_experts_grad", "experts": 64, "tokens": 4096,
         "top_k": 8, "m": 2048, "n": 768},
    ]


def _size(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]: half of the larger ones
    multiples of 128 (model widths), the others any size, odd ones included."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v >= 256 and rng.random() < 0.5:
        v = 128 * round(v / 128)
    return max(lo, min(hi, v))


def draw(rng):
    """One more case: norms of 1 to 65536 rows of 16 to 16384 values, routers
    of 1 to 65536 tokens and 4 to 512 experts, products of 1 to 8192 tokens and
    64 to 14336 a side, banks of 2 to 64 experts of 64 to 2048 a side."""
    kind = rng.choice(["norm", "norm_grad", "route", "route_grad", "mx4_bank", "mx4_linear", "mx4_experts",
                       "mx4_experts_grad"])
    if kind.startswith("norm"):
        rows, cols = _size(rng, 1, 65536), _size(rng, 16, 16384)
        return {"kind": kind, "rows": max(1, min(rows, (1 << 26) // cols)), "cols": cols,
                "dtype": rng.choice(["bf16", "fp32"]), "pad": rng.choice([0, 0, 1, 8])}
    if kind.startswith("route"):
        experts = _size(rng, 4, 512)
        tokens = min(_size(rng, 1, 65536), (1 << 22) // experts)
        return {"kind": kind, "tokens": tokens, "experts": experts, "top_k": rng.randint(1, min(8, experts)),
                "dtype": rng.choice(["bf16", "fp32"]), "masked": rng.choice([0.0, 0.1]),
                "renorm": rng.random() < 0.5}
    if kind == "mx4_linear":
        return {"kind": kind, "tokens": _size(rng, 1, 8192), "m": _size(rng, 64, 4096), "n": _size(rng, 64, 14336)}
    experts, m, n = _size(rng, 2, 64), _size(rng, 64, 2048), _size(rng, 64, 2048)
    if kind == "mx4_bank":
        return {"kind": kind, "batch": experts, "m": m, "n": min(n, (1 << 26) // (experts * m) or 1)}
    return {"kind": kind, "experts": experts, "tokens": _size(rng, 1, 4096), "top_k": rng.randint(1, min(8, experts)),
            "m": m, "n": n}


# ----------------------------------------------------------------- inputs
def _dtype(case):
    return torch.bfloat16 if case.get("dtype", "bf16") == "bf16" else torch.float32


def _generator(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * int(seed) + what)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _activations(g, rows, cols):
    """Hidden states: unit values, an offset of each row, a few strong channels."""
    x = _randn(g, rows, cols)
    strong = torch.rand(cols, generator=g, device="cuda") < 0.01
    return x * torch.where(strong, 8.0, 1.0) + 0.5 * _randn(g, rows, 1)


def _grads(g, rows, cols):
    """Gradients of rows: small, of sizes that differ from row to row."""
    return _randn(g, rows, cols) * (1e-4 * torch.exp(_randn(g, rows, 1)))


def _strided(x, pad, dtype):
    """x as the left part of a tensor that is `pad` columns wider."""
    if not pad:
        return x.to(dtype)
    wide = torch.zeros(x.shape[0], x.shape[1] + pad, device="cuda", dtype=dtype)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _padded(k):
    return -(-k // 256) * 256


def _capacity(tokens, experts, top_k):
    """Rows of a dispatch plan, whatever the routing: each expert padded to 32."""
    return -(-(tokens * top_k + 31 * min(experts, tokens * top_k)) // 32) * 32


def _pack(x):
    """fp32 [..., rows, k] in packed MXFP4 along k: (data, scale) bytes."""
    k = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, _padded(k) - k))
    code, e = _codes(x)
    data = code[..., 0::2] | (code[..., 1::2] << 4)
    return data.contiguous(), (e + 127).to(torch.uint8).contiguous()


def _codes(x):
    """4-bit codes (uint8, one a value) and block exponents of fp32 [..., 32 b]."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    e = _exponent(b)
    v = b * _two(-e[..., None])
    code = (_grid(v.abs())[..., None] > _levels(x)[:-1]).sum(-1).to(torch.uint8)
    return torch.where(v < 0, code | 8, code).reshape(x.shape), e


def _two(e):
    """2^e exactly, for whole e in [-127, 127] (pow need not be exact)."""
    return torch.where(e > -127, (e.int() + 127) << 23, 1 << 22).int().view(torch.float32)


def _levels(x):
    return torch.tensor(LEVELS, device=x.device, dtype=x.dtype)


def _exponent(blocks):
    """e of each block [..., 32]; -127 for a block of zeros."""
    amax = blocks.abs().amax(-1)
    return torch.where(amax > 0, torch.frexp(amax)[1] - 3, -127).clamp_min(-127)


def _grid(a):
    """|values| rounded to the 4-bit levels: steps of 0.5 below 2, 1 below 4, 2 above."""
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.round(a / step) * step).clamp_max(6.0)


def _routing(g, case):
    """A skewed routing of `tokens` to distinct experts, as the router's plan
    has it: offsets, row_token, and the most rows an expert has."""
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    index = (_randn(g, T, E) + 0.5 * _randn(g, E)).topk(k, dim=1).indices
    chosen = torch.zeros(T, E, dtype=torch.int64, device="cuda").scatter_(1, index, 1)
    counts = chosen.sum(0)
    ends = ((counts + 31) // 32 * 32).cumsum(0)
    offsets = torch.cat([ends.new_zeros(1), ends])
    position = (offsets[:-1] + chosen.t().contiguous().cumsum(1).t() - 1).gather(1, index)
    row_token = torch.full((_capacity(T, E, k),), -1, dtype=torch.int32, device="cuda")
    row_token[position] = torch.arange(T, dtype=torch.int32, device="cuda")[:, None]
    return {"offsets": offsets.int(), "row_token": row_token, "most": int(counts.max() + 31) // 32 * 32}


def prepare(case, seed):
    kind, g, s = case["kind"], _generator(seed, 1), {"case": case}
    dt = _dtype(case)
    if kind.startswith("norm"):
        rows, cols, pad = case["rows"], case["cols"], case["pad"]
        s["x"] = _strided(_activations(g, rows, cols), pad, dt)
        s["weight"] = 1 + 0.1 * _randn(g, cols)
        s["bias"] = 0.1 * _randn(g, cols)
        if kind == "norm_grad":
            s["dy"] = _strided(_grads(g, rows, cols), pad, dt)
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = 1 / ((x - s["mean"][:, None]).square().mean(1) + EPS).sqrt()
    elif kind.startswith("route"):
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        s["logits"] = (1.5 * _randn(g, T, E) + 0.7 * _randn(g, E)).to(dt)
        s["mask"] = torch.rand(T, generator=g, device="cuda") >= case["masked"]
        if kind == "route_grad":
            index, _, chosen, _ = _choose(s["logits"].float(), s["mask"], k)
            s["index"] = index.int()
            s["counts"] = torch.cat([chosen.sum(0), s["mask"].sum()[None]]).int()
            s["dgate"] = 1e-3 * _randn(g, T, k)
            s["dloss"] = torch.tensor([0.5], device="cuda")
    elif kind == "mx4_bank":
        s["weight"] = 0.02 * _randn(g, case["batch"], case["m"], case["n"])
    elif kind == "mx4_linear":
        s["x"] = _activations(g, case["tokens"], case["m"]).to(dt)
        s["w"] = _pack(0.02 * _randn(g, case["n"], case["m"]))
    else:
        s.update(_routing(g, case))
        s["x"] = _activations(g, case["tokens"], case["m"]).to(dt)
        if kind == "mx4_experts":
            s["w"] = _pack(0.02 * _randn(g, case["experts"], case["n"], case["m"]))
        else:
            s["dy"] = (_grads(g, s["row_token"].numel(), case["n"]) * (s["row_token"] >= 0)[:, None]).to(dt)
    return s


# ------------------------------------------------------------- plain forms
def _choose(l, mask, k):
    """(index or -1, row routes, chosen [T, E], p) of fp32 logits: the k largest
    of a row, ties to the lowest index."""
    order = torch.sort(l, dim=1, descending=True, stable=True).indices[:, :k]
    index = torch.where(mask[:, None], order, -1)
    chosen = torch.zeros(l.shape, dtype=torch.int64, device=l.device).scatter_(1, order, 1) * mask[:, None]
    p = torch.exp(l - l.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True) * mask[:, None]
    return index, mask, chosen, p


def _route(s):
    c, l = s["case"], s["logits"].float()
    T, E, k = c["tokens"], c["experts"], c["top_k"]
    index, mask, chosen, p = _choose(l, s["mask"], k)
    gate = p.gather(1, index.clamp_min(0)) * mask[:, None]
    if c["renorm"]:
        gate = torch.where(mask[:, None], gate / gate.sum(1, keepdim=True), 0.0)
    counts, n = chosen.sum(0), mask.sum()
    share = counts.float() / counts.sum().clamp_min(1)
    loss = BALANCE * E * (share * p.sum(0) / n.clamp_min(1)).sum()
    ends = ((counts + 31) // 32 * 32).cumsum(0)
    offsets = torch.cat([ends.new_zeros(1), ends])
    position = (offsets[:-1] + chosen.t().contiguous().cumsum(1).t() - 1).gather(1, index.clamp_min(0))
    position = torch.where(mask[:, None], position, -1)
    rows = _capacity(T, E, k)
    row_token = torch.full((rows + 1,), -1, dtype=torch.int32, device=l.device)
    token = torch.arange(T, dtype=torch.int32, device=l.device)[:, None].expand(T, k)
    row_token[torch.where(mask[:, None], position, rows)] = token
    return {"index": index.int(), "gate": gate, "counts": torch.cat([counts, n[None]]).int(), "loss": loss.view(1),
            "offsets": offsets.int(), "position": position.int(), "row_token": row_token[:rows]}


def _route_grad(s):
    c, l, k = s["case"], s["logits"].float(), s["case"]["top_k"]
    E, mask, index = c["experts"], s["mask"], s["index"].long()
    p = torch.exp(l - l.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    counts, n = s["counts"][:-1], s["counts"][-1]
    b = s["dloss"] * BALANCE * E * (counts.float() / counts.sum().clamp_min(1)) / n.clamp_min(1)
    at, dgate = index.clamp_min(0), s["dgate"] * (index >= 0)
    if c["renorm"]:
        gate = p.gather(1, at) * (index >= 0)
        gate = gate / gate.sum(1, keepdim=True).clamp_min(1e-30)
        part = gate * (dgate - (gate * dgate).sum(1, keepdim=True))
        dl = p * (b - (p * b).sum(1, keepdim=True))
        dl = dl.scatter_add(1, at, part)
    else:
        d = b.expand(l.shape).scatter_add(1, at, dgate)
        dl = p * (d - (p * d).sum(1, keepdim=True))
    return {"dlogits": torch.where(mask[:, None], dl, 0.0).to(s["logits"].dtype)}


def _quantised(x):
    """The values that fp32 [..., k] has in MXFP4 along k."""
    k = x.shape[-1]
    b = torch.nn.functional.pad(x, (0, -k % 32)).unflatten(-1, (-1, 32))
    e = _exponent(b)[..., None]
    v = b * _two(-e)
    v = torch.copysign(_grid(v.abs()), v)
    return (v * _two(e)).flatten(-2)[..., :k]


def _unpacked(packed, k):
    """fp32 values [..., k] of packed (data, scale) bytes."""
    data, scale = packed
    code = torch.stack([data & 15, data >> 4], -1).flatten(-2).long()
    level = torch.tensor(LEVELS, device=data.device)[code & 7]
    v = torch.where(code > 7, -level, level).unflatten(-1, (-1, 32))
    return (v * _two(scale.int()[..., None] - 127)).flatten(-2)[..., :k]


def _groups(s):
    """Rows of each expert [E, most] and which of them are its own."""
    o = s["offsets"].long()
    at = torch.arange(s["most"], device=o.device)
    return o[:-1, None] + at, at < (o[1:] - o[:-1])[:, None]


def _dispatched(s):
    rows = s["row_token"].long()
    return s["x"].float()[rows.clamp_min(0)] * (rows >= 0)[:, None]


def _plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind.startswith("norm"):
        x = s["x"].float()
        if kind == "norm":
            mean = x.mean(1)
            rstd = 1 / ((x - mean[:, None]).square().mean(1) + EPS).sqrt()
            y = (x - mean[:, None]) * rstd[:, None] * s["weight"] + s["bias"]
            return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}
        dy = s["dy"].float()
        h = (x - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["weight"]
        dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        return {"dx": dx.to(s["x"].dtype), "dweight": (dy * h).sum(0), "dbias": dy.sum(0)}
    if kind == "route":
        return _route(s)
    if kind == "route_grad":
        return _route_grad(s)
    if kind == "mx4_bank":
        w = s["weight"]
        return {"along_n": _quantised(w).bfloat16(), "along_m": _quantised(w.transpose(1, 2)).bfloat16()}
    if kind == "mx4_linear":
        return {"y": (_quantised(s["x"].float()) @ _unpacked(s["w"], c["m"]).t()).bfloat16()}
    at, mine = _groups(s)
    at = at.clamp_max(s["row_token"].numel() - 1)
    if kind == "mx4_experts":
        x = _quantised(_dispatched(s))[at] * mine[..., None]
        y = x @ _unpacked(s["w"], c["m"]).transpose(1, 2)
        out = torch.zeros(s["row_token"].numel(), c["n"], device="cuda", dtype=torch.bfloat16)
        out[at[mine]] = y[mine].bfloat16()
        return {"y": out}
    x = _quantised(_dispatched(s).t()).t()[at] * mine[..., None]
    dy = _quantised(s["dy"].float().t()).t()[at] * mine[..., None]
    return {"dw": x.transpose(1, 2) @ dy}


# -------------------------------------------------------- the package's own
def _own(s):
    import paper_2607_20548_amd as soap
    c = s["case"]
    kind = c["kind"]
    if kind.startswith("norm"):
        norm = s.get("norm")
        if norm is None:
            norm = s["norm"] = soap.LayerNorm(s["weight"], s["bias"], eps=EPS)
        if kind == "norm":
            y, mean, rstd = norm.forward(s["x"])
            return {"y": y, "mean": mean, "rstd": rstd}
        dx, dweight, dbias = norm.backward(s["dy"], s["x"], s["mean"], s["rstd"])
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    if kind.startswith("route"):
        router = s.get("router")
        if router is None:
            router = s["router"] = soap.Router(c["experts"], c["top_k"], renormalize=c["renorm"], balance=BALANCE)
        if kind == "route":
            r = router.forward(s["logits"], s["mask"])
            return {"index": r.index, "gate": r.gate, "counts": r.counts, "loss": r.loss, "offsets": r.offsets,
                    "position": r.position, "row_token": r.row_token}
        return {"dlogits": router.backward(s["logits"], s["index"], s["counts"], s["dgate"], s["dloss"],
                                           mask=s["mask"])}
    if kind == "mx4_bank":
        along_n, along_m = soap.mx4_quantize(s["weight"], along="both")
        return {"along_n": along_n.values(torch.bfloat16), "along_m": along_m.values(torch.bfloat16)}
    if kind == "mx4_linear":
        w = soap.Mx4(*s["w"], c["m"])
        return {"y": soap.mx4_product(soap.mx4_quantize(s["x"]), w, dtype=torch.bfloat16)}
    if kind == "mx4_experts":
        x = soap.mx4_quantize(s["x"], row_index=s["row_token"])
        return {"y": soap.mx4_product_rows(x, soap.Mx4(*s["w"], c["m"]), s["offsets"], dtype=torch.bfloat16)}
    x = soap.mx4_quantize(s["x"], row_index=s["row_token"], along="rows")
    dy = soap.mx4_quantize(s["dy"], along="rows")
    return {"dw": soap.mx4_product_k(x, dy, s["offsets"])}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    kind = case["kind"]
    size = 2.0 if case.get("dtype", "bf16") == "bf16" else 4.0
    mx = 17.0 / 32.0                                  # packed bytes of a value
    if kind.startswith("norm"):
        r, c = case["rows"], case["cols"]
        if kind == "norm":
            return {"bytes": 2 * size * r * c + 8 * r + 8 * c, "flops": 8.0 * r * c}
        return {"bytes": 3 * size * r * c + 8 * r + 12 * c, "flops": 15.0 * r * c}
    if kind.startswith("route"):
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        if kind == "route":
            rows = _capacity(T, E, k)
            return {"bytes": size * T * E + T + 12 * T * k + 4 * rows + 8 * E, "flops": (6.0 + k) * T * E}
        return {"bytes": 2 * size * T * E + T + 8 * T * k + 4 * E, "flops": 10.0 * T * E}
    m, n = case["m"], case["n"]
    if kind == "mx4_bank":
        count = float(case["batch"]) * m * n
        return {"bytes": (4 + 2 * 2) * count, "flops": 6.0 * count}
    if kind == "mx4_linear":
        T = case["tokens"]
        return {"bytes": 2.0 * T * m + mx * m * n + 2.0 * T * n, "flops": 2.0 * T * m * n}
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    routed = T * k
    if kind == "mx4_experts":
        return {"bytes": 2.0 * T * m + mx * min(E, routed) * m * n + 2.0 * routed * n, "flops": 2.0 * routed * m * n}
    return {"bytes": 2.0 * T * m + 2.0 * routed * n + 4.0 * E * m * n, "flops": 2.0 * routed * m * n}


# ---------------------------------------------- the same from 64-bit formulas
def _exact_mx4(x):
    """MXFP4 values along the last axis, from the definition: the nearest
    level, of two equally near ones that with the even code."""
    x = x.double()
    k = x.shape[-1]
    b = torch.nn.functional.pad(x, (0, -k % 32)).unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1, keepdim=True)
    two = _exact_powers(torch.floor(torch.log2(torch.where(amax > 0, amax, 1.0))) - 2)
    a = b.abs() / two
    q = torch.zeros_like(a)
    for code in range(1, 8):
        middle = (LEVELS[code - 1] + LEVELS[code]) / 2
        up = a >= middle if code % 2 == 0 else a > middle
        q = torch.where(up, torch.full_like(q, LEVELS[code]), q)
    return (torch.sign(b) * q * two).flatten(-2)[..., :k]


def _exact_powers(e):
    table = torch.tensor([math.ldexp(1.0, i) for i in range(-160, 128)], dtype=torch.float64, device=e.device)
    return table[e.long() + 160]


def _exact_unpack(packed, k):
    data, scale = packed
    table = torch.tensor(LEVELS + [-v for v in LEVELS], device=data.device, dtype=torch.float64)
    v = torch.empty(*data.shape[:-1], 2 * data.shape[-1], dtype=torch.float64, device=data.device)
    v[..., 0::2] = table[(data % 16).long()]
    v[..., 1::2] = table[(data // 16).long()]
    return (v * _exact_powers(scale.long() - 127).repeat_interleave(32, -1))[..., :k]


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind.startswith("norm"):
        x, w = s["x"].double(), s["weight"].double()
        if kind == "norm":
            var, mean = torch.var_mean(x, dim=1, correction=0)
            rstd = torch.rsqrt(var + EPS)
            return {"y": torch.addcmul(s["bias"].double(), (x - mean[:, None]) * rstd[:, None], w), "mean": mean,
                    "rstd": rstd}
        # the gradient for the mean and rstd that the call is given
        dy, r = s["dy"].double(), s["rstd"].double()[:, None]
        h = (x - s["mean"].double()[:, None]) * r
        cols = case["cols"]
        dh = dy * w
        dx = (r / cols) * (cols * dh - dh.sum(1, keepdim=True) - h * (dh * h).sum(1, keepdim=True))
        return {"dx": dx, "dweight": torch.einsum("rc,rc->c", dy, h), "dbias": dy.sum(0)}
    if kind.startswith("route"):
        l, mask, E, k = s["logits"].double(), s["mask"], case["experts"], case["top_k"]
        p = torch.softmax(l, 1)
        if kind == "route":
            top = torch.sort(l, dim=1, descending=True, stable=True).indices[:, :k]
            top = top[mask]
            gate = torch.zeros(case["tokens"], k, dtype=torch.float64, device="cuda")
            pick = p[mask].gather(1, top)
            gate[mask] = pick / pick.sum(1, keepdim=True) if case["renorm"] else pick
            counts = torch.bincount(top.reshape(-1), minlength=E).double()
            n = max(1, int(mask.sum()))
            loss = BALANCE * E * torch.dot(counts / max(1.0, float(counts.sum())), p[mask].sum(0) / n)
            return {"index": None, "gate": gate, "counts": None, "loss": loss.view(1), "offsets": None,
                    "position": None, "row_token": None}
        l.requires_grad_(True)
        p = torch.softmax(l, 1)
        live = s["index"] >= 0
        gate = p.gather(1, s["index"].long().clamp_min(0))
        if case["renorm"]:
            gate = gate / gate.sum(1, keepdim=True)
        counts = s["counts"].double()
        n, chosen = counts[-1].clamp_min(1), counts[:-1].sum().clamp_min(1)
        loss = BALANCE * E * ((counts[:-1] / chosen) * (p * mask[:, None]).sum(0) / n).sum()
        total = (gate * s["dgate"].double() * live).sum() + s["dloss"].double()[0] * loss
        return {"dlogits": torch.autograd.grad(total, l)[0]}
    if kind == "mx4_bank":
        w = s["weight"]
        return {"along_n": _exact_mx4(w), "along_m": _exact_mx4(w.mT)}
    if kind == "mx4_linear":
        return {"y": _exact_mx4(s["x"]) @ _exact_unpack(s["w"], case["m"]).mT}
    o, rows = s["offsets"].tolist(), s["row_token"].long()
    x = torch.where((rows >= 0)[:, None], s["x"].double()[rows.clamp_min(0)], 0.0)
    if kind == "mx4_experts":
        x, w = _exact_mx4(x), _exact_unpack(s["w"], case["m"])
        y = torch.zeros(rows.numel(), case["n"], dtype=torch.float64, device="cuda")
        for e in range(case["experts"]):
            y[o[e]:o[e + 1]] = x[o[e]:o[e + 1]] @ w[e].mT
        return {"y": y}
    x, dy = _exact_mx4(x.mT), _exact_mx4(s["dy"].mT)
    return {"dw": torch.stack([x[:, o[e]:o[e + 1]] @ dy[:, o[e]:o[e + 1]].mT for e in range(case["experts"])])}
