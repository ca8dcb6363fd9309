"""Trains one layer of experts: layer norm, router, the experts' products in MXFP4,
and the bank's update by one batched Muon (or SOAP) step.

    python examples/expert_layer.py                       # a small layer, 30 steps
    python examples/expert_layer.py --tokens 4096 --experts 64 --top-k 8 --m 2048 --n 768

The layer maps tokens of m values to n:  y_t = sum_j gate_tj W[e_tj]^T norm(x_t), the
experts e_tj and gates being the router's choice.  It learns the outputs of a random
layer of the same kind.  The weights, statistics, gates and gradients of parameters are
fp32, activations bfloat16; the three products of every expert (forward, input gradient,
weight gradient) take both operands in MXFP4 and sum in fp32, so the weight gradient
arrives as the [experts][m][n] bank that the batched steps read.
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


def matmul(a, b, trans_a=False, trans_b=False):
    """op(a) op(b) of contiguous fp32 matrices."""
    m, k = (a.shape[1], a.shape[0]) if trans_a else a.shape
    n = b.shape[0] if trans_b else b.shape[1]
    out = a.new_empty((m, n))
    soap.soap_gemm_f32(int(trans_a), int(trans_b), m, n, k, 1.0, a, a.shape[1], b, b.shape[1], 0.0, out, n)
    return out


class ExpertLayer:
    def __init__(self, experts, top_k, m, n, seed=0, optimizer="muon", lr=0.02, balance=0.01):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.weight, self.bias = torch.ones(m, device="cuda"), torch.zeros(m, device="cuda")
        self.route = 0.5 * m ** -0.5 * randn(m, experts)
        self.bank = m ** -0.5 * randn(experts, m, n)
        self.router = soap.Router(experts, top_k, renormalize=True, balance=balance)
        self.lr, self.t, self.optimizer = lr, 0, optimizer
        if optimizer == "muon":
            self.state = soap.MuonState(m, n, batch=experts)
        else:
            self.state = soap.SoapState(m, n, batch=experts)
        self.pack()

    def pack(self):
        """The bank in MXFP4 for both products that read it: blocks along n for the input
        gradient, along m (transposed) for the forward product."""
        self.along_n, self.along_m = soap.mx4_quantize(self.bank, along="both")

    def forward(self, x):
        """y float32 [tokens, n]; keeps what the backward pass needs."""
        norm = soap.LayerNorm(self.weight, self.bias)
        h, mean, rstd = norm.forward(x)
        hf = h.float()
        logits = matmul(hf, self.route)
        r = self.router.forward(logits)
        rows = soap.mx4_product_rows(soap.mx4_quantize(h, row_index=r.row_token), self.along_m, r.offsets,
                                     torch.bfloat16).float()
        picked = rows[r.position.long()]                       # [tokens, top_k, n]
        y = (picked * r.gate[..., None]).sum(1)
        self.kept = (x, norm, mean, rstd, h, hf, logits, r, picked)
        return y

    def backward(self, dy):
        """Gradients of the loss with gradient dy (float32 [tokens, n]) plus the balance loss."""
        x, norm, mean, rstd, h, hf, logits, r, picked = self.kept
        at = r.position.long()
        dgate = (picked * dy[:, None]).sum(-1)
        # every row's gradient: its token's, times its gate; zeros where a row has no token
        row_gate = dy.new_zeros(r.row_token.numel())
        row_gate[at.view(-1)] = r.gate.view(-1)
        drows = (dy[r.row_token.long().clamp_min(0)] * row_gate[:, None]).bfloat16()
        along_cols, along_rows = soap.mx4_quantize(drows, along="both")
        dbank = soap.mx4_product_k(soap.mx4_quantize(h, row_index=r.row_token, along="rows"), along_rows, r.offsets)
        dh = soap.mx4_product_rows(along_cols, self.along_n, r.offsets, torch.bfloat16).float()[at].sum(1)
        dlogits = self.router.backward(logits, r.index, r.counts, dgate)
        dh += matmul(dlogits, self.route, trans_b=True)
        droute = matmul(hf, dlogits, trans_a=True)
        dx, dweight, dbias = norm.backward(dh.bfloat16(), x, mean, rstd)
        return {"x": dx, "weight": dweight, "bias": dbias, "route": droute, "bank": dbank}

    def step(self, grads):
        """The bank by its batched optimizer step, the rest by plain gradient descent."""
        self.t += 1
        if self.optimizer == "muon":
            # a step of the polar factor moves every singular value by lr sqrt(max(m, n))
            self.state.step(self.bank, grads["bank"], COEFFS, beta1=0.9, lr=self.lr / max(self.bank.shape[1:]),
                            weight_decay=0.0)
        else:
            self.state.step(self.bank, grads["bank"], self.t, lr=self.lr / 10, weight_decay=0.0)
        for p, name in ((self.weight, "weight"), (self.bias, "bias"), (self.route, "route")):
            p -= self.lr * grads[name]
        self.pack()


def train(tokens, experts, top_k, m, n, steps, seed=0, optimizer="muon", lr=0.2, report=lambda *a: None):
    """The mean square errors of the steps, learning a layer of another seed."""
    teacher = ExpertLayer(experts, top_k, m, n, seed=seed + 1)
    layer = ExpertLayer(experts, top_k, m, n, seed=seed, optimizer=optimizer, lr=lr)
    layer.route.copy_(teacher.route)                           # the same split of the tokens
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    x = torch.randn(tokens, m, generator=g, device="cuda").bfloat16()
    target = teacher.forward(x)
    losses = []
    for t in range(steps):
        start = time.perf_counter()
        err = layer.forward(x) - target
        loss = err.square().mean()
        layer.step(layer.backward(2.0 / err.numel() * err))
        losses.append(loss.item())
        counts = layer.kept[7].counts
        report(t, losses[-1], layer.kept[7].loss.item(), int(counts[:-1].min()), int(counts[:-1].max()),
               time.perf_counter() - start)
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("tokens", 512), ("experts", 16), ("top-k", 2), ("m", 256), ("n", 128), ("steps", 30)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--optimizer", choices=["muon", "soap"], default="muon")
    ap.add_argument("--lr", type=float, default=0.2)
    a = ap.parse_args()
    train(a.tokens, a.experts, a.top_k, a.m, a.n, a.steps, optimizer=a.optimizer, lr=a.lr,
          report=lambda t, loss, balance, lo, hi, s: print(
              f"step {t + 1:3d}  error {loss:.5f}  balance loss {balance:.5f}  tokens of an expert {lo} to {hi}  "
              f"{1e3 * s:.1f} ms", flush=True))


if __name__ == "__main__":
    main()
