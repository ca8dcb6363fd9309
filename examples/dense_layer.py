"""Trains one dense layer and its classifier from a teacher's top classes: layer norm, heads'
norm and rotation, attention, gated feed-forward, distillation, and Muon (or SOAP) steps of
the weights.

    python examples/dense_layer.py                        # a small layer, 30 steps
    python examples/dense_layer.py --batch 8 --length 1024 --m 2048 --n 8192 --heads 16 --kv-heads 4 --classes 32000

    a = x + attention(turn(norm(q)), turn(norm(k)), v) W_o      q, k, v = norm(x) W_qkv
    y = a + (silu(norm(a) W_gate) * (norm(a) W_up)) W_down
    logits = norm(y) W_out

It learns the logits of a random layer of the same kind, of which it sees the largest of every
token.  Weights, the norms' gradients and gradients of weights are fp32; activations and the
products' operands bfloat16.  Attention itself and the plain products are torch's.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_20548_amd as soap  # noqa: E402

# Newton-Schulz triples of Muon: the Taylor quintic of the polar factor
COEFFS = [(15 / 8, -5 / 4, 3 / 8)] * 5
BF = torch.bfloat16


def attention(q, k, v, past=0):
    """Causal attention in fp32 of [batch, length, heads, dim], heads of k and v shared by runs of
    q's; the first query stands at position `past` of k and v."""
    share = q.shape[2] // k.shape[2]
    q, k, v = (t.transpose(1, 2).contiguous() for t in (q, k.repeat_interleave(share, 2), v.repeat_interleave(share, 2)))
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * q.shape[3] ** -0.5
    at = past + torch.arange(q.shape[2], device=q.device)
    later = torch.arange(k.shape[2], device=q.device)[None, :] > at[:, None]
    return torch.matmul(scores.masked_fill(later, float("-inf")).softmax(3), v).transpose(1, 2)


def weight_grad(x, dy):
    return x.float().t() @ dy.float()


class DenseLayer:
    """Matrices are fp32 `weights`, "in" x "out", with bfloat16 copies in `w`; vectors fp32."""

    def __init__(self, m, n, heads, kv_heads, dim, classes, seed=0, optimizer="muon", lr=0.02):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: s[-2] ** -0.5 * torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.weights = {"qkv": randn(m, (heads + 2 * kv_heads) * dim), "o": randn(heads * dim, m),
                        "gate_up": randn(2, m, n), "down": randn(n, m), "out": randn(m, classes)}
        ones = lambda n: torch.ones(n, device="cuda")  # noqa: E731
        self.vectors = {"norm1": ones(m), "norm2": ones(m), "norm3": ones(m), "q": ones(dim), "k": ones(dim)}
        self.bias = torch.zeros(m, device="cuda")
        self.optimizer, self.lr, self.t = optimizer, lr, 0
        state = soap.MuonState if optimizer == "muon" else soap.SoapState
        self.states = {name: state(*w.shape[-2:], batch=w.numel() // (w.shape[-2] * w.shape[-1]))
                       for name, w in self.weights.items()}
        self.cast()

    def cast(self):
        self.w = {name: w.to(BF) for name, w in self.weights.items()}
        v = self.vectors
        self.norms = [soap.LayerNorm(v["norm%d" % i], self.bias) for i in (1, 2, 3)]
        self.turn = soap.HeadNorm(self.dim, v["q"], v["k"])
        self.block = soap.GatedFeedForward(self.w["gate_up"][0], self.w["gate_up"][1], self.w["down"])

    def split(self, qkv):
        """Queries, keys and values: views of [tokens, heads, dim] into the fused rows."""
        return qkv.view(qkv.shape[0], -1, self.dim).split([self.heads, self.kv_heads, self.kv_heads], 1)

    def forward(self, x, batch, past=None):
        """logits [tokens, classes] of batch sequences' tokens in turn, x bfloat16 [tokens, m].  With
        `past`, a list of (keys, values) [batch, length, kv heads, dim], x holds the tokens that
        follow; it gets theirs.  Keeps what the backward pass needs."""
        shape = lambda t: t.view(batch, -1, *t.shape[1:])  # noqa: E731
        start = past[0].shape[1] if past else 0
        positions = (start + torch.arange(x.shape[0] // batch, device=x.device, dtype=torch.int32)).repeat(batch)
        h1, *s1 = self.norms[0].forward(x)
        q, k, v = self.split(h1 @ self.w["qkv"])
        tq, tk = self.turn.forward(q, k, positions)
        keys, values = shape(tk), shape(v)
        if past is not None:
            if past:
                keys, values = torch.cat([past[0], keys], 1), torch.cat([past[1], values], 1)
            past[:] = keys, values
        heads = [t.float().requires_grad_(past is None) for t in (shape(tq), keys, values)]
        with torch.set_grad_enabled(past is None):
            out = attention(*heads, past=start)
        o = out.detach().reshape(x.shape[0], -1).to(BF)
        a = x + o @ self.w["o"]
        h2, *s2 = self.norms[1].forward(a)
        f, gate, up = self.block.forward(h2, keep=past is None)
        y = a + f
        h3, *s3 = self.norms[2].forward(y)
        self.kept = (x, positions, h1, s1, q, k, heads, out, o, a, h2, s2, gate, up, y, h3, s3)
        return h3 @ self.w["out"]

    def backward(self, dlogits):
        """Gradients of matrices and vectors, and of x, from that of the last forward's logits."""
        x, positions, h1, s1, q, k, heads, out, o, a, h2, s2, gate, up, y, h3, s3 = self.kept
        grads = {"out": weight_grad(h3, dlogits)}
        dy, grads["norm3"], _ = self.norms[2].backward(dlogits @ self.w["out"].t(), y, *s3)
        dh2, dgate, dup, grads["down"] = self.block.backward(dy, h2, gate, up)
        grads["gate_up"] = torch.stack([dgate, dup])
        da, grads["norm2"], _ = self.norms[1].backward(dh2, a, *s2)
        da += dy
        grads["o"] = weight_grad(o, da)
        dout = (da @ self.w["o"].t()).float().view(out.shape)
        dtq, dtk, dv = (g.reshape(x.shape[0], -1, self.dim).to(BF) for g in torch.autograd.grad(out, heads, dout))
        dq, dk, grads["q"], grads["k"] = self.turn.backward(dtq, dtk, q, k, positions)
        dqkv = torch.cat([dq, dk, dv], 1).view(x.shape[0], -1)
        grads["qkv"] = weight_grad(h1, dqkv)
        dx, grads["norm1"], _ = self.norms[0].backward(dqkv @ self.w["qkv"].t(), x, *s1)
        grads["x"] = dx + da
        return grads

    def step(self, grads):
        """The matrices by their optimizer step, the vectors by plain gradient descent."""
        self.t += 1
        for name, w in self.weights.items():
            if self.optimizer == "muon":
                # a step of the polar factor moves every singular value by lr sqrt(max(m, n))
                self.states[name].step(w, grads[name], COEFFS, beta1=0.9, lr=self.lr / max(w.shape[-2:]), weight_decay=0.0)
            else:
                self.states[name].step(w, grads[name], self.t, lr=self.lr / 10, weight_decay=0.0)
        for name, v in self.vectors.items():
            v -= self.lr * grads[name]
        self.cast()


def train(batch, length, m, n, heads, kv_heads, dim, classes, top_k, steps, seed=0, optimizer="muon", lr=0.2,
          temperature=2.0, report=lambda *a: None):
    """The mean losses of the steps, learning from a layer of another seed."""
    teacher = DenseLayer(m, n, heads, kv_heads, dim, classes, seed=seed + 1)
    layer = DenseLayer(m, n, heads, kv_heads, dim, classes, seed=seed, optimizer=optimizer, lr=lr)
    distill = soap.Distillation(temperature)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    x = torch.randn(batch * length, m, generator=g, device="cuda").to(BF)
    values, index = teacher.forward(x, batch, past=[]).topk(top_k, 1)
    mean = torch.full((batch * length,), 1.0 / (batch * length), device="cuda")
    losses = []
    for t in range(steps):
        start = time.perf_counter()
        loss, dlogits = distill.forward_backward(layer.forward(x, batch), index.int(), values, mean)
        layer.step(layer.backward(dlogits))
        losses.append(loss.mean().item())
        report(t, losses[-1], time.perf_counter() - start)
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in (("batch", 4), ("length", 128), ("m", 256), ("n", 512), ("heads", 4), ("kv-heads", 2), ("dim", 64),
                          ("classes", 1000), ("top-k", 16), ("steps", 30)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--optimizer", choices=["muon", "soap"], default="muon")
    ap.add_argument("--lr", type=float, default=0.2)
    train(**vars(ap.parse_args()), report=lambda t, loss, s: print(f"step {t + 1:3d}  loss {loss:.5f}  {1e3 * s:.1f} ms",
                                                                   flush=True))


if __name__ == "__main__":
    main()
