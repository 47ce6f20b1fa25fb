"""The oracle of the rotary positions and of the operators around a paged microscaled cache, in numpy and 64 bits (TEST INFRASTRUCTURE
ONLY; shares no code with the library).  One row, one pair and one key at a time, by the definitions in include/hago.h."""
from __future__ import annotations

import math

import numpy as np

from . import mx_ref


def rope(x, positions, frequencies, axes=None, interleaved=False):
    """x [T, heads, dim], positions [axes, T]; frequencies as they are given (binary32)."""
    y = x.astype(np.float64).copy()
    pairs = len(frequencies)
    for t in range(x.shape[0]):
        for j in range(pairs):
            angle = float(positions[0 if axes is None else axes[j]][t]) * float(frequencies[j])
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + pairs)
            c, s = math.cos(angle), math.sin(angle)
            y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            y[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
    return y


def blocks(dim):
    return -(-dim // 32)


def row_bytes(dim, fmt):
    return blocks(dim) * (16 if fmt == "fp4" else 32)


def encode_row(x, fmt):
    """Rows [n, dim] -> (codes as they lie in the cache, scales)."""
    codes, scales = mx_ref.encode(x, fmt)
    return codes[:, :row_bytes(x.shape[1], fmt)], scales[:, :blocks(x.shape[1])]


def decode_row(codes, scales, fmt, dim):
    return mx_ref.decode(codes, scales, fmt, dim)


class Sequences:
    def __init__(self, table, lengths, offsets, pages, page):
        self.table, self.lengths, self.offsets, self.pages, self.page = np.asarray(table), np.asarray(lengths), np.asarray(offsets), pages, page

    def row(self, t):
        """(sequence, position) of row t, or None."""
        for s in range(len(self.lengths)):
            if self.offsets[s] <= t < self.offsets[s + 1]:
                return s, int(self.lengths[s]) - int(self.offsets[s + 1]) + t
        return None

    def place(self, s, position):
        """(page, place in it), or None."""
        if position < 0 or position >= self.table.shape[1] * self.page:
            return None
        page = int(self.table[s, position // self.page])
        return (page, position % self.page) if 0 <= page < self.pages else None


def attention(q, k_of, v_of, seqs, scale, causal=True, window=0):
    """q [T, heads, dim]; k_of, v_of [pages, kv_heads, page, dim] in 64 bits.  Returns (out, lse, weight) where weight[t, h] is the average of |v| by
    the probabilities, [T, heads, dim], and spread the largest sum of |q k| of a row's keys times |scale|; NaN rows for rows in no sequence."""
    T, heads, dim = q.shape
    out = np.full((T, heads, dim), np.nan)
    lse = np.full((T, heads), np.nan)
    weight = np.zeros((T, heads, dim))
    spread = np.zeros((T, heads))
    group = heads // k_of.shape[1]
    for t in range(T):
        found = seqs.row(t)
        if found is None:
            continue
        s, p = found
        seen = [seqs.place(s, j) for j in range(max(0, int(seqs.lengths[s]))) if (not causal or j <= p) and (not window or j > p - window)]
        seen = [x for x in seen if x is not None]
        for h in range(heads):
            if not seen:
                out[t, h], lse[t, h] = 0.0, -np.inf
                continue
            pages, at = np.array(seen).T
            k, v = k_of[pages, h // group, at], v_of[pages, h // group, at]
            score = scale * (k @ q[t, h].astype(np.float64))
            e = np.exp(score - score.max())
            out[t, h] = e @ v / e.sum()
            lse[t, h] = score.max() + math.log(e.sum())
            weight[t, h] = e @ np.abs(v) / e.sum()
            spread[t, h] = abs(scale) * (np.abs(k) @ np.abs(q[t, h].astype(np.float64))).max()
    return out, lse, weight, spread
