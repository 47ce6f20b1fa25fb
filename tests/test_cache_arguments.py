"""What the rotary positions and the operators around a paged cache refuse, on the host and before anything is launched."""
import ctypes as C
import math
import os

import pytest
import torch

import paper_2103_14949_amd as hago
from paper_2103_14949_amd import binding


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(hago.library_path()):
        from paper_2103_14949_amd import build
        build.build()
    return hago.lib()


P = 0x1000   # an aligned pointer that is never followed
NULL, SHAPE, DTYPE, PARAM = 1, 2, 3, 5


def test_rope(L):
    def call(x=P, t=hago.BF16, T=4, heads=3, dim=64, row=192, head=64, pos=P, axes=1, freq=P, axis=None, pairs=32, order=0, out=4 * P, orow=192, ohead=64):
        return L.hago_rope(x, t, T, heads, dim, row, head, pos, axes, freq, axis, pairs, order, out, orow, ohead, None)
    assert call(x=None) == NULL and call(out=None) == NULL and call(pos=None) == NULL and call(freq=None) == NULL
    for bad in (dict(T=-1), dict(heads=-1), dict(dim=-1), dict(pairs=-1), dict(pairs=33), dict(axes=0), dict(dim=4097, head=5000, row=2 ** 16, ohead=5000, orow=2 ** 16),
                dict(heads=65537), dict(T=2 ** 31), dict(row=-1), dict(head=-1), dict(orow=-1), dict(ohead=-1), dict(row=2 ** 62), dict(head=2 ** 62),
                dict(ohead=63), dict(orow=191), dict(orow=0), dict(ohead=0), dict(orow=64, ohead=192)):
        assert call(**bad) == SHAPE, bad
    for t in (hago.U8, hago.I32, 8, -1):
        assert call(t=t) == DTYPE
    assert call(order=2) == PARAM and call(order=-1) == PARAM
    for bad in (dict(x=P + 1), dict(out=P + 1), dict(pos=P + 2), dict(freq=P + 1), dict(axis=P + 2), dict(t=hago.F32, x=P + 2)):
        assert call(**bad) == PARAM, bad
    assert call(out=P, row=200) == PARAM and call(out=P, head=65) == PARAM   # in place with other distances
    for nothing in (dict(T=0), dict(heads=0), dict(dim=0, pairs=0)):
        assert call(x=None, out=None, pos=None, freq=None, **nothing) == 0
    assert call(T=0, t=hago.U8) == DTYPE


def cache(**k):
    a = dict(kc=P, ks=P, vc=P, vs=P, kf=hago.MX_FP8, vf=hago.MX_FP4, pages=9, heads=2, page=16, dim=64)
    a.update(k)
    return binding._MxCache(*a.values())


def sequences(**k):
    a = dict(table=P, lengths=P, offsets=P, seqs=3, cols=4, stride=4)
    a.update(k)
    return binding._MxSequences(*a.values())


def write(L, c=None, s=None, k=P, krow=128, khead=64, v=P, vrow=128, vhead=64, t=hago.BF16, T=5, kv=None, vv=None):
    return L.hago_mx_cache_write(C.byref(c or cache()), C.byref(s or sequences()), k, krow, khead, v, vrow, vhead, t, T, kv, vv, None)


def read(L, c=None, s=None, t=hago.BF16, T=5, k=P, v=P):
    return L.hago_mx_cache_read(C.byref(c or cache()), C.byref(s or sequences()), t, T, k, v, None)


def attend(L, c=None, s=None, q=P, t=hago.BF16, T=5, heads=4, row=256, head=64, scale=0.1, causal=1, window=0, out=P, lse=None, ws=P, bytes=None):
    if bytes is None:
        bytes = 1 << 40
    return L.hago_mx_attention(C.byref(c or cache()), C.byref(s or sequences()), q, t, T, heads, row, head, scale, causal, window, out, lse, ws, bytes, None)


@pytest.mark.parametrize("call", [write, read, attend])
def test_caches_and_sequences(L, call):
    for bad in (dict(kc=None), dict(ks=None), dict(vc=None), dict(vs=None)):
        assert call(L, c=cache(**bad)) == NULL, bad
    for bad in (dict(table=None), dict(lengths=None), dict(offsets=None)):
        assert call(L, s=sequences(**bad)) == NULL, bad
    for bad in (dict(pages=-1), dict(pages=2 ** 31), dict(heads=-1), dict(heads=65537), dict(page=0), dict(page=-1), dict(page=2 ** 31), dict(dim=-1), dict(dim=257),
                dict(pages=2 ** 31 - 1, heads=65536, page=2 ** 29)):
        assert call(L, c=cache(**bad)) == SHAPE, bad
    for bad in (dict(seqs=-1), dict(seqs=2 ** 31), dict(cols=-1), dict(stride=3), dict(cols=2 ** 28, stride=2 ** 28), dict(stride=2 ** 62)):
        assert call(L, s=sequences(**bad)) == SHAPE, bad
    assert call(L, T=-1) == SHAPE and call(L, T=2 ** 31) == SHAPE
    for t in (hago.U8, hago.I32, 8, -1):
        assert call(L, t=t) == DTYPE
    for bad in (dict(kf=2), dict(vf=-1), dict(kc=P + 8), dict(vc=P + 8)):
        assert call(L, c=cache(**bad)) == PARAM, bad
    for bad in (dict(table=P + 2), dict(lengths=P + 2), dict(offsets=P + 1)):
        assert call(L, s=sequences(**bad)) == PARAM, bad
    assert call(L, T=0) == 0 and call(L, s=sequences(seqs=0, table=None, lengths=None, offsets=None)) == 0
    assert call(L, T=0, t=hago.U8) == DTYPE


def test_structs_are_wanted(L):
    assert L.hago_mx_cache_write(None, C.byref(sequences()), P, 128, 64, P, 128, 64, hago.BF16, 5, None, None, None) == NULL
    assert L.hago_mx_cache_read(C.byref(cache()), None, hago.BF16, 5, P, P, None) == NULL
    assert L.hago_mx_attention(None, None, P, hago.BF16, 5, 4, 256, 64, 0.1, 1, 0, P, None, P, 1 << 40, None) == NULL


def test_write_and_read(L):
    assert write(L, k=None) == NULL and write(L, v=None) == NULL and read(L, k=None) == NULL and read(L, v=None) == NULL
    for bad in (dict(krow=-1), dict(khead=-1), dict(vrow=-1), dict(vhead=-1), dict(krow=2 ** 61)):
        assert write(L, **bad) == SHAPE, bad
    for bad in (dict(k=P + 1), dict(v=P + 1), dict(kv=P + 1), dict(vv=P + 1), dict(t=hago.F32, k=P + 2)):
        assert write(L, **bad) == PARAM, bad
    assert read(L, k=P + 1) == PARAM and read(L, t=hago.F32, v=P + 2) == PARAM
    assert write(L, c=cache(heads=0), k=None, v=None) == 0 and write(L, c=cache(dim=0), k=None, v=None) == 0


def test_attention(L):
    bytes = L.hago_mx_attention_workspace_bytes
    assert bytes(5, 3, 4, 2, 64) > 0 and bytes(0, 3, 4, 2, 64) == 0 and bytes(1, 1, 8, 2, 256) > bytes(1, 1, 8, 2, 64) and bytes(5, 1000, 4, 2, 64) > bytes(5, 3, 4, 2, 64)
    for bad in ((-1, 3, 4, 2, 64), (5, -1, 4, 2, 64), (5, 3, -4, 2, 64), (5, 3, 4, -2, 64), (5, 3, 5, 2, 64), (5, 3, 4, 0, 64), (5, 3, 4, 2, 257), (2 ** 26, 3, 4, 2, 64),
                (5, 3, 4, 65537, 64), (5, 2 ** 21 + 1, 4, 2, 64)):
        assert bytes(*bad) == -1, bad
    assert attend(L, q=None) == NULL and attend(L, out=None) == NULL and attend(L, ws=None) == NULL
    for bad in (dict(heads=5), dict(heads=-4), dict(window=-1), dict(row=-1), dict(head=-1), dict(row=2 ** 61), dict(T=2 ** 26)):
        assert attend(L, **bad) == SHAPE, bad
    assert attend(L, s=sequences(seqs=2 ** 21 + 1)) == SHAPE
    for bad in (dict(scale=math.inf), dict(scale=math.nan), dict(scale=-2e30), dict(q=P + 1), dict(out=P + 1), dict(lse=P + 2), dict(ws=P + 128), dict(bytes=bytes(5, 3, 4, 2, 64) - 1)):
        assert attend(L, **bad) == PARAM, bad
    assert attend(L, heads=0, q=None, out=None, ws=None) == 0


def tensors(T=5, seqs=3):
    c = hago.MXCache.empty(9, 2, 16, 64, hago.MX_FP8, hago.MX_FP4, device="cpu")
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    return c, torch.zeros(T, 2, 64, dtype=torch.bfloat16), (i(seqs, 4), i(seqs), i(seqs + 1))


def edited(c, **k):
    return hago.MXCache(*[k.get(n, getattr(c, n)) for n in hago.MXCache.__slots__])


CACHE, X, WHERE = tensors()
Q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
POS, FREQ = torch.zeros(1, 5, dtype=torch.int32), torch.zeros(32)


@pytest.mark.parametrize("call,error", [
    (lambda: hago.rope(Q, POS, FREQ), AssertionError),   # host tensors
    (lambda: hago.rope(Q[0], POS, FREQ), AssertionError),
    (lambda: hago.rope(Q.double(), POS, FREQ), TypeError),
    (lambda: hago.rope(Q.transpose(1, 2), POS, FREQ), AssertionError),
    (lambda: hago.rope(Q, POS.long(), FREQ), AssertionError),
    (lambda: hago.rope(Q, POS[:, :4], FREQ), AssertionError),
    (lambda: hago.rope(Q, POS, FREQ.double()), AssertionError),
    (lambda: hago.rope(Q, POS, torch.zeros(33)), AssertionError),
    (lambda: hago.rope(Q, POS, FREQ, axes=torch.zeros(31, dtype=torch.int32)), AssertionError),
    (lambda: hago.rope(Q, POS, FREQ, out=Q.float()), AssertionError),
    (lambda: hago.rope(Q, POS, FREQ, out=Q[:4]), AssertionError),
    (lambda: hago.rope(Q, None, FREQ), TypeError),
    (lambda: hago.mx_cache_write(CACHE, X, X, *WHERE), AssertionError),
    (lambda: hago.mx_cache_write(edited(CACHE, k_fmt=hago.MX_FP4), X, X, *WHERE), AssertionError),
    (lambda: hago.mx_cache_write(edited(CACHE, k_fmt=7), X, X, *WHERE), AssertionError),
    (lambda: hago.mx_cache_write(edited(CACHE, v_scales=CACHE.v_scales[:8]), X, X, *WHERE), AssertionError),
    (lambda: hago.mx_cache_write(edited(CACHE, v_scales=CACHE.v_scales.float()), X, X, *WHERE), AssertionError),
    (lambda: hago.mx_cache_write(edited(CACHE, k_codes=CACHE.k_codes[:, :, ::2]), X, X, *WHERE), AssertionError),
    (lambda: hago.mx_cache_write(edited(CACHE, dim=96), X, X, *WHERE), AssertionError),
    (lambda: hago.mx_cache_write(CACHE, X, X[:4], *WHERE), AssertionError),
    (lambda: hago.mx_cache_write(CACHE, X, X.half(), *WHERE), AssertionError),
    (lambda: hago.mx_cache_write(CACHE, Q, Q, *WHERE), AssertionError),
    (lambda: hago.mx_cache_write(CACHE, X, X, WHERE[0].long(), *WHERE[1:]), AssertionError),
    (lambda: hago.mx_cache_write(CACHE, X, X, WHERE[0], WHERE[1][:2], WHERE[2]), AssertionError),
    (lambda: hago.mx_cache_write(CACHE, X, X, WHERE[0], WHERE[1], WHERE[1]), AssertionError),
    (lambda: hago.mx_cache_write(None, X, X, *WHERE), AttributeError),
    (lambda: hago.mx_cache_read(CACHE, *WHERE, -1), AssertionError),
    (lambda: hago.mx_cache_read(CACHE, *WHERE, 5, out_dtype=77), KeyError),
    (lambda: hago.mx_cache_read(CACHE, *WHERE, 5, out=X), AssertionError),
    (lambda: hago.mx_cache_read(CACHE, *WHERE, 5, out=(X, X.float())), AssertionError),
    (lambda: hago.mx_cache_read(CACHE, *WHERE, 5), AssertionError),
    (lambda: hago.mx_attention(Q, CACHE, *WHERE), AssertionError),
    (lambda: hago.mx_attention(Q[:, :3], CACHE, *WHERE), AssertionError),
    (lambda: hago.mx_attention(Q[..., :32], CACHE, *WHERE), AssertionError),
    (lambda: hago.mx_attention(Q, CACHE, *WHERE, scale="x"), TypeError),
    (lambda: hago.mx_attention(Q, CACHE, *WHERE, out=Q.float()), AssertionError),
    (lambda: hago.mx_attention(Q, CACHE, *WHERE, lse=torch.zeros(5, 3)), AssertionError),
    (lambda: hago.mx_attention(Q, CACHE, *WHERE, workspace=torch.zeros(64, dtype=torch.uint8)), AssertionError),
])
def test_the_binding_refuses(L, call, error):
    with pytest.raises(error):
        call()
