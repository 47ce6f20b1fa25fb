"""Performance cases of the operators around a paged cache of keys and values that is held on microscaled codes: what a program
that serves a quantized transformer has them do between the products of its layers.

    rope       x[T, heads, dim], positions[axes, T]   -> x with pairs of columns turned by position * frequency
    write      k, v[T, kv_heads, dim]                 -> their codes and scales in the pages of their sequences
    read       rows of sequences                      -> the values that their codes stand for
    attention  q[T, heads, dim] over the cache        -> softmax(scale * q k) v, each row over its sequence's keys

Codes are E2M1 (fp4, two a byte) or E4M3 (fp8) in blocks of 32 columns that share a power-of-two scale of 8 bits (E8M0); a block of
largest magnitude m has the scale 2^(floor(log2 m) - emax), emax 2 or 8.  A page holds [kv_heads, page, blocks * 32] codes and
[kv_heads, page, blocks] scales, zero codes behind column dim.  Sequence s owns the pages table[s], has lengths[s] tokens with the
new ones, and its new tokens are rows offsets[s] .. offsets[s + 1] of the call: row i of n has position lengths[s] - n + i.  A
query at position p sees the keys 0 .. p (all of its sequence's where it is not causal), with a window w only those behind p - w.
"""
from __future__ import annotations

import math
import random

import torch

DEV = "cuda:0"
own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
FP4_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


# ---------------------------------------------------------------- the cases

def listed():
    layer = dict(heads=32, kv_heads=8, dim=128, page=64)
    return [
        # Queries and keys of one token far behind the start, side by side in the result of one product.
        dict(name="rope_token", kind="rope", T=1, heads=40, rest=8, dim=128, pairs=64, axes=1, interleaved=False, far=131072, type="bf16"),
        # Image and video positions (time, height, width) in rows of no convenient size, neighbours paired, some columns not turned.
        dict(name="rope_three_axes", kind="rope", T=4001, heads=20, rest=10, dim=80, pairs=33, axes=3, interleaved=True, far=3000, type="f16"),
        # Queries and keys of a long prompt.
        dict(name="rope_prompt", kind="rope", T=8192, heads=40, rest=8, dim=128, pairs=64, axes=1, interleaved=False, far=8192, type="bf16"),
        # A serving batch's step: one token of each of 64 sequences goes into the cache.
        dict(name="write_tokens", kind="write", seqs=64, new_min=1, new=1, length_min=1024, length=16384, layout=1, k_fmt="fp8", v_fmt="fp8", type="bf16",
             values=False, **layer),
        # Four prompts go into the cache; a simulation of the quantized model goes on with the values.
        dict(name="write_prompts", kind="write", seqs=4, new_min=1500, new=3000, length_min=1500, length=3000, layout=2, k_fmt="fp8", v_fmt="fp4", type="bf16",
             values=True, **layer),
        # Sequences of odd lengths read back, a head dimension of two and a half blocks, pages that are no power of two.
        dict(name="read_odd_sizes", kind="read", seqs=7, new_min=1, new=2500, length_min=1, length=2500, layout=3, kv_heads=5, heads=15, dim=80, page=48,
             k_fmt="fp8", v_fmt="fp4", type="f16"),
        # A long document's cache for a program that works on the real values.
        dict(name="read_document", kind="read", seqs=1, new_min=131072, new=131072, length_min=131072, length=131072, layout=4, k_fmt="fp8", v_fmt="fp8",
             type="bf16", **layer),
        # One user, one token: latency.
        dict(name="attend_token", kind="attention", seqs=1, new_min=1, new=1, length_min=1000, length=1000, layout=5, k_fmt="fp8", v_fmt="fp8", type="bf16",
             causal=True, window=0, **layer),
        # A serving batch's step over sequences of very different lengths.
        dict(name="attend_tokens", kind="attention", seqs=64, new_min=1, new=1, length_min=1024, length=16384, layout=6, k_fmt="fp8", v_fmt="fp8", type="bf16",
             causal=True, window=0, **layer),
        # Odd sizes throughout: short and long chunks together, a window, keys in 8 bits and values in 4.
        dict(name="attend_odd_sizes", kind="attention", seqs=5, new_min=1, new=97, length_min=1, length=1500, layout=7, heads=15, kv_heads=5, dim=80, page=48,
             k_fmt="fp8", v_fmt="fp4", type="f16", causal=True, window=300),
        # A chunk of a long document whose beginning the cache holds.
        dict(name="attend_chunk", kind="attention", seqs=1, new_min=1024, new=1024, length_min=32768, length=32768, layout=8, k_fmt="fp8", v_fmt="fp4",
             type="bf16", causal=True, window=0, **layer),
        # A long prompt from its first token on.
        dict(name="attend_prompt", kind="attention", seqs=1, new_min=8192, new=8192, length_min=8192, length=8192, layout=9, k_fmt="fp8", v_fmt="fp8",
             type="bf16", causal=True, window=0, **layer),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above; every size is drawn over its whole range, odd ones included."""
    kind = rng.choice(["rope", "write", "read", "attention", "attention", "attention"])
    dim = rng.choice([64, 128, 128, 256, rng.randint(16, 256)])
    type = rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])
    if kind == "rope":
        heads = _log_int(rng, 1, 64)
        most = 8192 * 40 * 128 // (heads * dim) // (2 if type == "f32" else 1)
        return dict(kind=kind, T=max(1, min(_log_int(rng, 1, 16384), most)), heads=heads, rest=rng.choice([0, 1, heads // 4]), dim=dim,
                    pairs=rng.choice([dim // 2, dim // 2, dim // 4, rng.randint(1, dim // 2)]), axes=rng.choice([1, 1, 2, 3]),
                    interleaved=rng.random() < 0.4, far=_log_int(rng, 1, 1 << 20), type=type)
    kv_heads = rng.choice([1, 2, 4, 8, 8, rng.randint(1, 16)])
    heads = kv_heads * rng.choice([1, 2, 4, 4, 8, rng.randint(1, 16)])
    layer = dict(heads=heads, kv_heads=kv_heads, dim=dim, page=rng.choice([16, 32, 64, 64, 128, 256, rng.randint(1, 300)]), layout=rng.randint(0, 1 << 20),
                 k_fmt=rng.choice(["fp8", "fp8", "fp4"]), v_fmt=rng.choice(["fp8", "fp8", "fp4"]))
    seqs = _log_int(rng, 1, 128)
    row = kv_heads * _blocks(dim) * 32
    if kind in ("write", "read"):
        most = max(1, (8192 if kind == "write" else 65536) * 1024 // row // seqs // (2 if type == "f32" else 1))
        longest = min(_log_int(rng, 1, 65536), most)
        fewest = rng.choice([longest, rng.randint(1, longest)])
        if kind == "read":
            return dict(kind=kind, seqs=seqs, new_min=fewest, new=longest, length_min=fewest, length=longest, type=type, **layer)
        return dict(kind=kind, seqs=seqs, new_min=fewest, new=longest, length_min=longest, length=longest + rng.choice([0, 0, 1000]), type=type,
                    values=rng.random() < 0.4, **layer)
    # at most the bytes of the listed batch's cache, and the products of the listed prompt
    longest = min(_log_int(rng, 1, 131072), max(1, 64 * 5000 * 1024 // row // seqs))
    new = rng.choice([1, 1, _log_int(rng, 1, 8192)])
    new = max(1, min(new, longest, 8192 * 40 * 128 // (seqs * heads * dim), 8192 * 4096 * 32 * 128 // (longest * seqs * heads * dim * (6 if type == "f32" else 1))))
    fewest = rng.choice([longest, max(new, longest // 10)])
    return dict(kind=kind, seqs=seqs, new_min=rng.choice([new, 1]), new=new, length_min=fewest, length=longest, type=type, causal=rng.random() < 0.8,
                window=rng.choice([0, 0, 0, _log_int(rng, 1, longest)]), **layer)


def _sequences(case):
    """New tokens and lengths of the sequences, spread over the logarithm as a batch that users come to and leave."""
    rng = random.Random(case["layout"])
    lengths = [_log_int(rng, case["length_min"], case["length"]) for _ in range(case["seqs"])]
    whole = (case["new_min"], case["new"]) == (case["length_min"], case["length"])  # (all of it is new)
    return [n if whole else min(n, _log_int(rng, case["new_min"], case["new"])) for n in lengths], lengths


# ---------------------------------------------------------------- the inputs

def _blocks(dim):
    return (dim + 31) // 32


def _row_bytes(dim, fmt):
    return _blocks(dim) * (16 if fmt == "fp4" else 32)


def _pack(codes, fmt):
    """Codes, one a byte -> as they lie in memory: 4-bit ones two a byte, the even column in the lower half."""
    return codes if fmt == "fp8" else codes[..., 0::2] | codes[..., 1::2] << 4


def _pages(gen, pages, kv_heads, page, dim, fmt, outliers):
    """Codes and scales of pages whose tokens are a layer's keys (a few columns many times larger) or values."""
    codes = torch.empty(pages, kv_heads, page, _row_bytes(dim, fmt), dtype=torch.uint8, device=DEV)
    scales = torch.empty(pages, kv_heads, page, _blocks(dim), dtype=torch.uint8, device=DEV)
    gain = torch.where(torch.rand(kv_heads, 1, dim, generator=gen, device=DEV) < outliers, 6.0, 1.0)
    step = max(1, (1 << 25) // (kv_heads * page * dim))
    for first in range(0, pages, step):
        n = min(step, pages - first)
        x = torch.randn(n, kv_heads, page, dim, generator=gen, device=DEV) * gain
        c, s, _ = _encode(x.view(-1, dim), fmt)
        codes[first:first + n] = _pack(c, fmt).view(n, kv_heads, page, -1)
        scales[first:first + n] = s.view(n, kv_heads, page, -1)
    return codes, scales


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kind, s, dtype = case["kind"], dict(case), TYPES[case["type"]]
    dim = case["dim"]
    if kind == "rope":
        T, pairs = case["T"], case["pairs"]
        # (the columns that are not turned are the values, which the same product makes)
        s["x"] = torch.randn(T, case["heads"] + case["rest"], dim, generator=gen, device=DEV).to(dtype)[:, :case["heads"]]
        s["positions"] = torch.randint(0, case["far"], (case["axes"], T), generator=gen, device=DEV, dtype=torch.int32)
        if case["axes"] == 1:
            s["positions"] = (torch.arange(T, device=DEV, dtype=torch.int32) + max(0, case["far"] - T))[None]
        s["frequencies"] = torch.pow(10000.0, -torch.arange(pairs, device=DEV, dtype=torch.float64) / pairs).float()
        s["axis"] = (torch.arange(pairs, device=DEV) * case["axes"] // pairs).to(torch.int32) if case["axes"] > 1 else None
        return s
    new, lengths = _sequences(case)
    kv_heads, page = case["kv_heads"], case["page"]
    s["new"], s["total"], s["long"] = new, sum(new), lengths
    need = [(n + page - 1) // page for n in lengths]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.zeros(len(new), max(need) + 2, dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    s["table"] = table
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32).to(DEV)
    s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), torch.tensor(new).cumsum(0)]).to(torch.int32).to(DEV)
    if kind == "write":
        for x in "kv":
            s[x + "_codes"] = torch.zeros(pages, kv_heads, page, _row_bytes(dim, case[x + "_fmt"]), dtype=torch.uint8, device=DEV)
            s[x + "_scales"] = torch.zeros(pages, kv_heads, page, _blocks(dim), dtype=torch.uint8, device=DEV)
        # (keys and values as parts of one product's result)
        qkv = torch.randn(sum(new), case["heads"] + 2 * kv_heads, dim, generator=gen, device=DEV).to(dtype)
        s["k"], s["v"] = qkv[:, case["heads"]:case["heads"] + kv_heads], qkv[:, case["heads"] + kv_heads:]
        return s
    s["k_codes"], s["k_scales"] = _pages(gen, pages, kv_heads, page, dim, case["k_fmt"], 0.02)
    s["v_codes"], s["v_scales"] = _pages(gen, pages, kv_heads, page, dim, case["v_fmt"], 0.0)
    if kind == "attention":
        s["q"] = torch.randn(sum(new), case["heads"], dim, generator=gen, device=DEV).to(dtype)
    return s


# ---------------------------------------------------------------- the plain forms

def _encode(x, fmt):
    """x in 32 bits -> codes (one a byte) and scales in whole blocks of 32 columns, and the values they stand for [rows, cols]."""
    rows, cols = x.shape
    wide = torch.zeros(rows, _blocks(cols) * 32, device=x.device)
    wide[:, :cols] = x
    blocks = wide.view(rows, -1, 32)
    emax, low, bits, top = (2, 0, 1, 6.0) if fmt == "fp4" else (8, -6, 3, 448.0)
    largest = blocks.abs().amax(-1, keepdim=True)
    shared = torch.where(largest > 0, torch.frexp(largest)[1] - 1 - emax, -127).clamp(min=-127)
    scaled = torch.ldexp(torch.ldexp(blocks, -(shared // 2)), -(shared - shared // 2))  # (2^127 and more in two steps)
    size = scaled.abs()
    step = torch.ldexp(torch.ones_like(size), torch.where(size > 0, torch.frexp(size)[1] - 1, low).clamp(min=low) - bits)
    size = (torch.round(size / step) * step).clamp(max=top)
    grid = torch.tensor(FP4_VALUES, device=x.device) if fmt == "fp4" else torch.arange(127, dtype=torch.uint8, device=x.device).view(torch.float8_e4m3fn).float()
    codes = torch.searchsorted(grid, size).to(torch.uint8) + (torch.signbit(scaled) * (8 if fmt == "fp4" else 128)).to(torch.uint8)
    values = torch.ldexp(torch.ldexp(torch.copysign(size, scaled), shared // 2), shared - shared // 2)
    return codes.view(rows, -1), (shared[..., 0] + 127).to(torch.uint8), values.view(rows, -1)[:, :cols]


def _decode(codes, scales, fmt, cols):
    """Codes as they lie in memory, and scales -> the values, 32 bits [..., cols]."""
    if fmt == "fp4":
        lut = torch.tensor(FP4_VALUES + [-v for v in FP4_VALUES], device=codes.device)
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
        values = lut[codes.int()]
    else:
        values = codes.view(torch.float8_e4m3fn).float()
    scale = torch.exp2(scales.float() - 127)
    return (values.view(*scales.shape, 32) * scale[..., None]).flatten(-2)[..., :cols]


def _places(s):
    """Page and place in it of every row of the call."""
    page = s["page"]
    sequence = torch.repeat_interleave(torch.arange(len(s["new"]), device=DEV), torch.diff(s["offsets"]).long(), output_size=s["total"])
    at = torch.arange(s["total"], device=DEV) - s["offsets"].long()[1:][sequence] + s["lengths"].long()[sequence]
    return s["table"].long()[sequence, at // page], at % page


def _run_plain(s):
    kind, dtype, dim = s["kind"], TYPES[s["type"]], s["dim"]
    if kind == "rope":
        x, pairs = s["x"].float(), s["pairs"]
        axis = torch.zeros(pairs, dtype=torch.int64, device=DEV) if s["axis"] is None else s["axis"].long()
        angle = s["positions"].double()[axis].t() * s["frequencies"].double()  # [T, pairs]
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        first, second = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if s["interleaved"] else (slice(0, pairs), slice(pairs, 2 * pairs))
        y = x.clone()
        y[..., first] = x[..., first] * cos - x[..., second] * sin
        y[..., second] = x[..., second] * cos + x[..., first] * sin
        return y.to(dtype)
    if kind == "write":
        out, (pages, at) = {}, _places(s)
        for x in "kv":
            codes, scales, values = _encode(s[x].float().reshape(-1, dim), s[x + "_fmt"])
            s[x + "_codes"][pages, :, at] = _pack(codes, s[x + "_fmt"]).view(s["total"], s["kv_heads"], -1)
            s[x + "_scales"][pages, :, at] = scales.view(s["total"], s["kv_heads"], -1)
            out[x + "_codes"], out[x + "_scales"] = s[x + "_codes"], s[x + "_scales"]
            if s["values"]:
                out[x + "_values"] = values.view(s["total"], s["kv_heads"], dim).to(dtype)
        return out
    if kind == "read":
        pages, at = _places(s)
        return tuple(_decode(s[x + "_codes"][pages, :, at], s[x + "_scales"][pages, :, at], s[x + "_fmt"], dim).to(dtype) for x in "kv")
    out = torch.empty_like(s["q"])
    group, first = s["heads"] // s["kv_heads"], 0
    for i, (n, length) in enumerate(zip(s["new"], s["long"])):
        used = s["table"][i, :(length + s["page"] - 1) // s["page"]].long()
        key = torch.arange(length, device=DEV)
        at = torch.arange(length - n, length, device=DEV)[:, None]
        hidden = torch.zeros(n, length, dtype=torch.bool, device=DEV)
        if s["causal"]:
            hidden |= key > at
        if s["window"]:
            hidden |= key <= at - s["window"]
        for h in range(s["kv_heads"]):
            k, v = (_decode(s[x + "_codes"][used, h], s[x + "_scales"][used, h], s[x + "_fmt"], dim).view(-1, dim)[:length] for x in "kv")
            q = s["q"][first:first + n, h * group:(h + 1) * group].float() * dim ** -0.5
            score = (q.reshape(-1, dim) @ k.t()).view(n, group, length).masked_fill_(hidden[:, None], -math.inf)
            p = torch.exp(score - score.amax(-1, keepdim=True))
            y = (p.view(-1, length) @ v).view(n, group, dim) / p.sum(-1, keepdim=True)
            out[first:first + n, h * group:(h + 1) * group] = y.to(dtype)
        first += n
    return out


# ---------------------------------------------------------------- the framework's operators

def _run_own(s):
    import paper_2103_14949_amd as hago
    kind = s["kind"]
    if kind == "rope":
        return hago.rope(s["x"], s["positions"], s["frequencies"], axes=s["axis"], interleaved=s["interleaved"])
    formats = {"fp4": hago.MX_FP4, "fp8": hago.MX_FP8}
    cache = hago.MXCache(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], formats[s["k_fmt"]], formats[s["v_fmt"]], s["dim"])
    where = (s["table"], s["lengths"], s["offsets"])
    if kind == "write":
        values = hago.mx_cache_write(cache, s["k"], s["v"], *where, values=s["values"])
        out = {x + t: s[x + t] for x in "kv" for t in ("_codes", "_scales")}
        return {**out, "k_values": values[0], "v_values": values[1]} if s["values"] else out
    if kind == "read":
        return hago.mx_cache_read(cache, *where, s["total"], out_dtype={"bf16": hago.BF16, "f16": hago.F16, "f32": hago.F32}[s["type"]])
    return hago.mx_attention(s["q"], cache, *where, scale=s["dim"] ** -0.5, causal=s["causal"], window=s["window"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- the work

def work(case):
    size, dim = TYPES[case["type"]].itemsize, case["dim"]
    if case["kind"] == "rope":
        n = case["T"] * case["heads"] * dim
        return {"bytes": 2 * n * size + 4 * case["axes"] * case["T"] + 4 * case["pairs"], "flops": 3 * case["T"] * case["heads"] * 2 * case["pairs"]}
    new, lengths = _sequences(case)
    total, heads = sum(new), case["kv_heads"]
    token = heads * (_row_bytes(dim, case["k_fmt"]) + _row_bytes(dim, case["v_fmt"]) + 2 * _blocks(dim))
    plan = 8 * case["seqs"] + 4
    if case["kind"] in ("write", "read"):
        real = 2 * total * heads * dim * size
        pages = sum((n - 1) // case["page"] - (n - m) // case["page"] + 1 for m, n in zip(new, lengths))
        return {"bytes": real * (2 if case.get("values") else 1) + total * token + 4 * pages + plan, "flops": 2 * total * heads * dim * (4 if case["kind"] == "write" else 1)}
    seen = products = pages = 0
    for n, length in zip(new, lengths):
        at = range(length - n, length)
        lows = [max(0, p - case["window"] + 1) if case["window"] else 0 for p in at]
        ends = [p + 1 if case["causal"] else length for p in at]
        products += sum(e - b for b, e in zip(lows, ends))
        seen += length - lows[0]
        pages += (length - 1) // case["page"] - lows[0] // case["page"] + 1
    return {"bytes": 2 * total * case["heads"] * dim * size + seen * token + 4 * pages + plan, "flops": 4 * products * case["heads"] * dim}


# ---------------------------------------------------------------- the definition, in 64 bits

def _nearest(y, fmt):
    """Every y as the microscaled value that stands for it, by the definition: among the code values, the nearest one."""
    rows, cols = y.shape
    out = torch.empty_like(y)
    emax, exponents, mantissas, least = (2, range(0, 3), 2, 0) if fmt == "fp4" else (8, range(-6, 9), 8, -6)
    grid = [m / mantissas * 2.0 ** least for m in range(mantissas)]
    grid += [(1 + m / mantissas) * 2.0 ** e for e in exponents for m in range(mantissas)]
    grid = grid if fmt == "fp4" else grid[:-1]  # (the last one is no number)
    grid = torch.tensor(grid, dtype=torch.float64, device=y.device)
    between = (grid[1:] + grid[:-1]) / 2
    for first in range(0, cols, 32):
        block = y[:, first:first + 32]
        m = block.abs().amax(1, keepdim=True)
        e = torch.where(m > 0, torch.floor(torch.log2(torch.where(m > 0, m, 1.0))), -1000.0)
        e = torch.where(torch.pow(2.0, e) > m, e - 1, torch.where(torch.pow(2.0, e + 1) <= m, e + 1, e))  # (the logarithm is rounded)
        scale = torch.pow(2.0, (e - emax).clamp(min=-127.0))
        v = block.abs() / scale
        below = torch.searchsorted(between, v.contiguous(), right=False)  # ties: the lower one
        tie = (below < len(between)) & (between[below.clamp(max=len(between) - 1)] == v)
        code = below + (tie & (below % 2 == 1))
        out[:, first:first + 32] = torch.sign(block) * grid[code] * scale
    return out


def _number(codes, scales, fmt, cols):
    """The codes' values by their bits: sign, exponent, mantissa."""
    if fmt == "fp4":
        codes = torch.stack([codes % 16, codes // 16], -1).flatten(-2)
    mant, bias, sign = (1, 1, 8) if fmt == "fp4" else (3, 7, 128)
    c = torch.arange(2 * sign, device=codes.device)
    e, m = c % sign >> mant, (c % (1 << mant)).double() / (1 << mant)
    size = torch.where(e > 0, (1 + m) * torch.pow(2.0, (e - bias).double()), m * 2.0 ** (1 - bias))
    value = torch.where(c >= sign, -size, size)[codes.int()]
    return (value * torch.pow(2.0, scales.double() - 127).repeat_interleave(32, -1))[..., :cols]


def exact(case, seed):
    s = prepare(case, seed)
    kind, dim = case["kind"], case["dim"]
    if kind == "rope":
        x, pairs = s["x"].double(), case["pairs"]
        turns = torch.stack([s["positions"][0 if s["axis"] is None else int(s["axis"][j])].double() * s["frequencies"][j].double() for j in range(pairs)], -1)
        y = x.clone()
        for j in range(pairs):
            a, b = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + pairs)
            z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(turns[:, j]), turns[:, j])[:, None]
            y[..., a], y[..., b] = z.real, z.imag
        return y
    if kind == "write":
        if not case["values"]:
            return None  # (whole numbers only)
        values = {x + "_values": _nearest(s[x].double().reshape(-1, dim), case[x + "_fmt"]).view(s[x].shape) for x in "kv"}
        return {**{x + t: None for x in "kv" for t in ("_codes", "_scales")}, **values}
    parts = {"k": [], "v": []}
    out, first, group = [], 0, case["heads"] // case["kv_heads"]
    for i, (n, length) in enumerate(zip(s["new"], s["long"])):
        used = s["table"][i].long()[:-(-length // case["page"])]
        by_head = []
        for h in range(case["kv_heads"]):
            k, v = (_number(s[x + "_codes"][used, h], s[x + "_scales"][used, h], case[x + "_fmt"], dim).flatten(0, 1)[:length] for x in "kv")
            if kind == "read":
                by_head.append((k[length - n:], v[length - n:]))
                continue
            p = torch.arange(length - n, length, device=DEV)
            low = (p + 1 - case["window"]).clamp(min=0) if case["window"] else torch.zeros_like(p)
            end = p + 1 if case["causal"] else torch.full_like(p, length)
            key = torch.arange(length, device=DEV)
            seen = (key >= low[:, None]) & (key < end[:, None])
            for g in range(group):
                score = (s["q"][first:first + n, h * group + g].double() @ k.t()) / math.sqrt(dim)
                by_head.append(torch.softmax(torch.where(seen, score, -math.inf), -1) @ v)
        if kind == "read":
            for x, t in zip("kv", zip(*by_head)):
                parts[x].append(torch.stack(t, 1))
        else:
            out.append(torch.stack(by_head, 1))
        first += n
    return tuple(torch.cat(parts[x]) for x in "kv") if kind == "read" else torch.cat(out)
