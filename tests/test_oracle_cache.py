"""The oracle of the rotary positions and of the paged cache, pinned by closed forms and invariants."""
import numpy as np

from oracle import cache_ref as ref


def test_rope_turns_and_keeps_lengths():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 7))
    pos = np.array([[0, 1, 2], [5, 0, 9]])
    freq = np.array([np.pi / 2, 0.25, 1.0], np.float32)
    for interleaved in (False, True):
        y = ref.rope(x, pos, freq, [0, 1, 1], interleaved)
        pairs = [(0, 1), (2, 3), (4, 5)] if interleaved else [(0, 3), (1, 4), (2, 5)]
        assert np.array_equal(y[..., 6], x[..., 6])
        for j, (a, b) in enumerate(pairs):
            z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * np.asarray(pos[[0, 1, 1][j]] * np.float64(freq[j])))[:, None]
            assert np.allclose(y[..., a], z.real, atol=1e-15) and np.allclose(y[..., b], z.imag, atol=1e-15)
    assert np.allclose(ref.rope(x, pos * 0, freq), x)


def test_places():
    s = ref.Sequences([[4, 9, -1], [1, 0, 2]], [25, 7], [2, 5, 6], 9, 10)
    assert [s.row(t) for t in range(7)] == [None, None, (0, 22), (0, 23), (0, 24), (1, 6), None]
    assert s.place(0, 3) == (4, 3) and s.place(0, 13) is None and s.place(0, 23) is None   # a page that is not there, and -1
    assert s.place(1, 29) == (2, 9) and s.place(1, 30) is None and s.place(1, -1) is None


def test_attention_of_equal_keys_is_the_average():
    rng = np.random.default_rng(2)
    k, v = np.ones((4, 1, 3, 5)), rng.standard_normal((4, 1, 3, 5))
    seqs = ref.Sequences([[2, 0, 3, 1]], [11], [0, 3], 4, 3)
    flat = v[[2, 0, 3, 1], 0].reshape(-1, 5)
    out, lse, _, _ = ref.attention(rng.standard_normal((3, 2, 5)) * 0 + 0.5, k, v, seqs, 2.0)
    for i in range(3):
        assert np.allclose(out[i], flat[:9 + i].mean(0)) and np.allclose(lse[i], 5.0 + np.log(9 + i))
    out, _, _, _ = ref.attention(np.ones((3, 2, 5)), k, v, seqs, 1.0, window=2)
    assert np.allclose(out[0], flat[7:9].mean(0)) and np.allclose(out[2], flat[9:11].mean(0))
    out, _, _, _ = ref.attention(np.ones((3, 2, 5)), k, v, seqs, 1.0, causal=False)
    assert np.allclose(out, flat[:11].mean(0))


def test_rows_that_see_nothing():
    seqs = ref.Sequences([[0]], [2], [0, 4], 1, 4)   # four rows of a sequence of two tokens: the first two stand before it
    out, lse, _, _ = ref.attention(np.ones((5, 1, 2)), np.ones((1, 1, 4, 2)), np.ones((1, 1, 4, 2)), seqs, 1.0)
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.allclose(out[2:4], 1) and np.isnan(out[4]).all()
