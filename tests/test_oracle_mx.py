"""Pins of the microscaled oracle: hand-worked codes, exact rationals, invariants, and the refusal of planted mistakes."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import mx_ref as mx


def test_code_values():
    assert mx.code_values("fp4").tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6]
    v = mx.code_values("fp8")
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[7] == 7 * 2.0 ** -9 and v[8] == 2.0 ** -6 and v[126] == 448 and np.isnan(v[[127, 255]]).all()
    assert v[0x38] == 1 and v[0x39] == 1.125 and v[0xC0] == -2
    assert np.array_equal(v[128:255], -v[:127])


@pytest.mark.parametrize("fmt,row,scale,want", [
    # largest magnitude 6: floor(log2 6) - 2 = 0.  2.5 is a tie of codes 4 and 5, 5 one of 6 and 7, .25 one of 0 and 1, 1.75 one of 3 and 4
    ("fp4", [6, 2.5, -5, .25, 1.75, .75, 3.5, -0.2], 127, [7, 4, 14, 0, 4, 2, 6, 8]),
    # largest magnitude just below 8: the same scale, saturated
    ("fp4", [7.9, -7, 1], 127, [7, 15, 2]),
    ("fp4", [0.0, -0.0], 0, [0, 8]),
    ("fp8", [448, 449, 1, -17, 2.0 ** -9, 2.0 ** -10], 127, [126, 126, 0x38, 0xD8, 1, 0]),   # -17: a tie of 16 and 18
    ("fp8", [1.0, 0.5], 119, [0x78, 0x70]),   # scale 2^-8: 256 and 128
])
def test_hand_worked_blocks(fmt, row, scale, want):
    codes, scales = mx.encode(np.array([row], np.float64), fmt)
    assert scales[0].tolist()[0] == scale and (scales[0][1:] == 0).all()
    assert mx.unpack(codes, fmt)[0, :len(row)].tolist() == want and (mx.unpack(codes, fmt)[0, len(row):] == 0).all()


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_codes_are_nearest_by_rationals(fmt):
    rng = np.random.default_rng(3)
    grid = [Fraction(v) for v in mx.code_values(fmt)[:8 if fmt == "fp4" else 127]]
    x = (rng.standard_normal((1, 32)) * 2.0 ** rng.integers(-30, 30, (1, 32))).astype(np.float32)
    codes, scales = mx.encode(x, fmt)
    codes = mx.unpack(codes, fmt)[0, :32]
    scale = Fraction(2) ** (int(scales[0, 0]) - 127)
    biggest = max(abs(Fraction(float(v))) for v in x[0])
    assert scale * 2 ** mx.EMAX[fmt] <= biggest < scale * 2 ** (mx.EMAX[fmt] + 1)
    for v, c in zip(x[0], codes):
        off = [abs(abs(Fraction(float(v))) / scale - g) for g in grid]
        best = min(off)
        assert off[c % (8 if fmt == "fp4" else 128)] == best
        assert off.count(best) == 1 or c % 2 == 0


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_values_encode_to_themselves(fmt):
    rng = np.random.default_rng(4)
    x = rng.standard_normal((5, 200)) * 7
    codes, scales = mx.encode(x, fmt)
    v = mx.decode(codes, scales, fmt, 200)
    again, same = mx.encode(v, fmt)
    assert np.array_equal(codes, again) and np.array_equal(scales, same)


def test_blocks_without_a_number():
    x = np.ones((1, 96))
    x[0, 3], x[0, 70] = np.nan, -np.inf
    codes, scales = mx.encode(x, "fp8")
    assert scales[0].tolist() == [255, 119, 255, 0] and np.isnan(mx.decode(codes, scales, "fp8", 96)[0, :32]).all()
    assert (mx.unpack(codes, "fp8")[0, :32] == 0).all()


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_accepts_takes_the_codes_and_refuses_mistakes(fmt):
    rng = np.random.default_rng(5)
    y = rng.standard_normal((4, 160))
    codes, scales = mx.encode(y, fmt)
    assert mx.accepts(codes, scales, y, 1e-6, fmt)
    wrong = codes.copy()
    wrong[2, 17] ^= 2
    assert not mx.accepts(wrong, scales, y, 1e-6, fmt)
    wrong = scales.copy()
    wrong[1, 2] += 1
    assert not mx.accepts(codes, wrong, y, 1e-6, fmt)
    wrong = codes.copy()
    wrong[0, 0] ^= 0x80
    assert not mx.accepts(wrong, scales, np.abs(y) + 1, 1e-6, fmt)


def test_norm_and_activation_by_hand():
    h, y = mx.rmsnorm(np.array([[3.0, 4.0]]), np.array([2.0, 1.0]), np.array([[0.0, 0.0]]), 0.0)
    assert h.tolist() == [[3, 4]] and np.allclose(y, [[6 / np.sqrt(12.5), 4 / np.sqrt(12.5)]], rtol=1e-15)
    assert np.allclose(mx.silu_mul(np.array([[0.0, np.log(3.0), 5.0, 2.0]])), [[0.0, np.log(3.0) * 0.75 * 2]], rtol=1e-15)
