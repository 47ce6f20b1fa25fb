"""A layer of attention served on microscaled codes: norm, one product for queries, keys and values, rotary positions, the cache, attention, the product back.

    residual, a = norm(x + residual)                     8-bit codes
    q | k | v   = a Wqkv^T                               one product
    q, k        = turned by their positions              in place, side by side
    cache       <- k, v                                  8-bit and 4-bit codes in the pages of their sequences
    y           = attention of q over the cache          every sequence's own tokens, those of earlier calls with them
    out         = y Wo^T

Weights are realized in 4 bits once.  A call takes the new tokens of any number of sequences: whole prompts, chunks, or a token each.  Run as a program it
serves two prompts and then single tokens, and says how far the results are from the same layer in binary32 on the weights before they were
quantized, over a cache of its own:  python examples/mx_attention_layer.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2103_14949_amd as hago  # noqa: E402


class AttentionLayer:
    """wqkv [(heads + 2 * kv_heads) * dim, width], wo [width, heads * dim], gamma [width]; a cache of `pages` pages."""

    def __init__(self, wqkv, wo, gamma, heads, kv_heads, pages, page=64, theta=10000.0, eps=1e-5):
        self.dim = wqkv.shape[0] // (heads + 2 * kv_heads)
        self.wqkv, self.wo = (hago.mx_quantize(w, hago.MX_FP4) for w in (wqkv, wo))
        self.gamma, self.heads, self.kv_heads, self.eps = gamma, heads, kv_heads, eps
        self.frequencies = torch.pow(theta, -torch.arange(self.dim // 2, device=wqkv.device, dtype=torch.float64) / (self.dim // 2)).float()
        self.cache = hago.MXCache.empty(pages, kv_heads, page, self.dim, hago.MX_FP8, hago.MX_FP4, device=wqkv.device)

    def __call__(self, x, residual, positions, table, lengths, offsets):
        """x, residual [tokens, width] bfloat16 -> (what the layer adds, the new residual).  Nothing here waits for the device."""
        a, residual = hago.mx_rmsnorm(x, self.gamma, residual, self.eps, hago.MX_FP8)
        qkv = hago.mx_dense(a, self.wqkv).view(x.shape[0], self.heads + 2 * self.kv_heads, self.dim)
        turned = qkv[:, :self.heads + self.kv_heads]
        hago.rope(turned, positions, self.frequencies, out=turned)
        k, v = qkv[:, self.heads:self.heads + self.kv_heads], qkv[:, self.heads + self.kv_heads:]
        hago.mx_cache_write(self.cache, k, v, table, lengths, offsets)
        y = hago.mx_attention(qkv[:, :self.heads], self.cache, table, lengths, offsets)
        return hago.mx_dense(hago.mx_quantize(y.view(x.shape[0], self.heads * self.dim), hago.MX_FP8), self.wo), residual


def plain(weights, x, residual, heads, kv_heads, theta=10000.0, eps=1e-5):
    """The same layer for one whole sequence in binary32, on the weights themselves."""
    wqkv, wo, gamma = (t.float() for t in weights)
    n, dim = x.shape[0], wqkv.shape[0] // (heads + 2 * kv_heads)
    h = x.float() + residual.float()
    a = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + eps) * gamma
    qkv = (a @ wqkv.t()).view(n, -1, dim).transpose(0, 1)
    angle = torch.arange(n, device=x.device, dtype=torch.float64)[:, None] * torch.pow(theta, -torch.arange(dim // 2, device=x.device, dtype=torch.float64) / (dim // 2))
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    first, second = qkv[:heads + kv_heads].chunk(2, -1)
    turned = torch.cat([first * cos - second * sin, second * cos + first * sin], -1)
    k, v = (t.repeat_interleave(heads // kv_heads, 0) for t in (turned[heads:], qkv[heads + kv_heads:]))
    score = (turned[:heads] @ k.transpose(1, 2).contiguous()) * dim ** -0.5
    p = torch.softmax(score.masked_fill(torch.ones(n, n, dtype=torch.bool, device=x.device).triu(1), -float("inf")), -1)
    return (p @ v).transpose(0, 1).reshape(n, -1) @ wo.t(), h


def make(width, heads, kv_heads, dim, device="cuda", seed=0):
    gen = torch.Generator(device=device).manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device=device)  # noqa: E731
    return ((normal((heads + 2 * kv_heads) * dim, width) * width ** -0.5).bfloat16(), (normal(width, heads * dim) * (heads * dim) ** -0.5).bfloat16(),
            (1 + 0.1 * normal(width)).bfloat16())


def serve(weights, heads, kv_heads, xs, residuals, cuts, page=64):
    """Sequences xs[i] [tokens, width] in steps: cuts[i] are the numbers of tokens that sequence i has given after each.  What the layer adds to each token."""
    device = xs[0].device
    need = [-(-len(x) // page) for x in xs]
    layer = AttentionLayer(*weights, heads, kv_heads, sum(need), page)
    table = torch.zeros(len(xs), max(need), dtype=torch.int32)
    pages = torch.randperm(sum(need), generator=torch.Generator().manual_seed(1)).to(torch.int32)
    for i, n in enumerate(need):
        table[i, :n] = pages[sum(need[:i]):sum(need[:i + 1])]
    table, outs = table.to(device), [[] for _ in xs]
    for step in range(len(cuts[0])):
        spans = [(c[step - 1] if step else 0, c[step]) for c in cuts]
        new = [b - a for a, b in spans]
        rows = lambda ts: torch.cat([t[a:b] for t, (a, b) in zip(ts, spans)])  # noqa: E731
        positions = torch.cat([torch.arange(a, b) for a, b in spans]).to(torch.int32).to(device)
        lengths = torch.tensor([b for _, b in spans], dtype=torch.int32).to(device)
        offsets = torch.tensor([0] + new).cumsum(0).to(torch.int32).to(device)
        out, _ = layer(rows(xs), rows(residuals), positions, table, lengths, offsets)
        for i, part in enumerate(out.split(new)):
            outs[i].append(part)
    return [torch.cat(o) for o in outs]


def main(width=1024, heads=8, kv_heads=2, dim=128):
    weights = make(width, heads, kv_heads, dim)
    gen = torch.Generator(device="cuda").manual_seed(1)
    xs, residuals = ([torch.randn(n, width, generator=gen, device="cuda").bfloat16() for n in (300, 171)] for _ in range(2))
    off = 0.0
    for name, cuts in (("prompts at once", [[300], [171]]), ("and then token by token", [list(range(290, 301)), list(range(161, 172))])):
        for out, x, r in zip(serve(weights, heads, kv_heads, xs, residuals, cuts), xs, residuals):
            want, _ = plain(weights, x, r, heads, kv_heads)
            off = float((out.float() - want).norm() / want.norm())
            print("%s, %d tokens: %.3f of the layer in 32 bits away" % (name, len(x), off))
    return off


if __name__ == "__main__":
    main()
