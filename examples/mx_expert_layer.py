"""A layer of experts served on microscaled codes: norm, routed products, gated activation, products back, weighted sum.

    residual, a = norm(x + residual)                       8-bit codes
    gate, up    = a[token] W1[e]^T                         rows in the order of their experts
    h           = silu(gate) * up                          8-bit codes
    y           = h W2[e]^T,  out[token] = sum of its experts' y by the router's weights

The weights are realized in 4 bits once.  Run as a program it serves a prompt and then single tokens and says how far the results are
from the same layer in binary32 on the weights before they were quantized:  python examples/mx_expert_layer.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2103_14949_amd as hago  # noqa: E402


def realize(w):
    """Weights [experts, features, inputs] -> their 4-bit codes."""
    e, n, k = w.shape
    mx = hago.mx_quantize(w.reshape(e * n, k), hago.MX_FP4)
    return hago.MX(mx.codes.view(e, n, -1), mx.scales.view(e, n, -1), hago.MX_FP4, k)


class ExpertLayer:
    """w1 [experts, 2 * hidden, width] (gate rows, then up rows), w2 [experts, width, hidden], router [experts, width], gamma [width]."""

    def __init__(self, w1, w2, router, gamma, top, eps=1e-5):
        self.w1, self.w2 = realize(w1), realize(w2)
        self.router, self.gamma, self.top, self.eps = router, gamma, top, eps
        self.experts = w1.shape[0]

    def __call__(self, x, residual):
        """x, residual [tokens, width] bfloat16 -> (what the layer adds, the new residual).  Nothing here waits for the device."""
        a, residual, normed = hago.mx_rmsnorm(x, self.gamma, residual, self.eps, hago.MX_FP8, values=True)
        weight, expert = torch.softmax(normed.float() @ self.router.float().t(), -1).topk(self.top, -1)
        weight = weight / weight.sum(-1, keepdim=True)
        # assignments in the order of their experts: which token each is made of, where each expert's begin
        order = torch.argsort(expert.flatten(), stable=True)
        token = (order // self.top).to(torch.int32)
        offsets = torch.searchsorted(expert.flatten()[order].contiguous(), torch.arange(self.experts + 1, device=x.device)).to(torch.int32)
        gate_up = hago.mx_dense_grouped(a, self.w1, offsets, rows=token)
        h = hago.mx_silu_mul(gate_up, hago.MX_FP8)
        y = hago.mx_dense_grouped(h, self.w2, offsets, out_dtype=hago.F32)
        out = torch.zeros(x.shape, dtype=torch.float32, device=x.device)
        back = torch.empty_like(order).scatter_(0, order, torch.arange(len(order), device=x.device)).view(-1, self.top)
        for k in range(self.top):   # one at a time, in the router's order, so that the sum is the same in every run
            out += weight[:, k, None] * y[back[:, k]]
        return out.to(x.dtype), residual


def plain(layer_weights, x, residual, top, eps=1e-5):
    """The same layer in binary32, on the weights themselves."""
    w1, w2, router, gamma = (t.float() for t in layer_weights)
    h = x.float() + residual.float()
    a = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + eps) * gamma
    weight, expert = torch.softmax(a @ router.t(), -1).topk(top, -1)
    weight = weight / weight.sum(-1, keepdim=True)
    out = torch.zeros_like(h)
    for e in range(w1.shape[0]):
        t, k = (expert == e).nonzero(as_tuple=True)
        gate, up = (a[t] @ w1[e].t()).chunk(2, -1)
        out.index_add_(0, t, weight[t, k, None] * ((torch.nn.functional.silu(gate) * up) @ w2[e].t()))
    return out, h


def make(experts, width, hidden, dtype=torch.bfloat16, device="cuda", seed=0):
    gen = torch.Generator(device=device).manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device=device)  # noqa: E731
    return ((normal(experts, 2 * hidden, width) * width ** -0.5).to(dtype), (normal(experts, width, hidden) * hidden ** -0.5).to(dtype),
            (normal(experts, width) * width ** -0.5).to(dtype), (1 + 0.1 * normal(width)).to(dtype))


def main(tokens=512, experts=16, width=1024, hidden=704, top=2):
    weights = make(experts, width, hidden)
    layer = ExpertLayer(*weights, top)
    gen = torch.Generator(device="cuda").manual_seed(1)
    stream = torch.randn(tokens, width, generator=gen, device="cuda").to(torch.bfloat16)
    for name, rows in (("prompt of %d tokens" % tokens, slice(0, tokens)), ("one token", slice(3, 4))):
        x = torch.randn(tokens, width, generator=gen, device="cuda").to(torch.bfloat16)[rows]
        out, residual = layer(x, stream[rows])
        want, h = plain(weights, x, stream[rows], top)
        off = (out.float() - want).norm() / want.norm()
        print("%s: %.3f of the layer in 32 bits away, residual %.4f" % (name, off, (residual.float() - h).norm() / h.norm()))
    return float(off)


if __name__ == "__main__":
    main()
