"""Pins of the oracle of the norm and the rotation by position: closed forms and invariants."""
import numpy as np

from oracle import rope


def test_by_hand():
    x = np.zeros((2, 1, 64))
    x[:, 0, 0], x[:, 0, 8], x[:, 0, 1], x[:, 0, 63] = 1.0, 2.0, 3.0, 5.0
    freq = np.zeros(8, dtype=np.float32)
    freq[0] = np.float32(0.5)
    y = rope.qk_norm_rope(x, None, 0.0, freq, np.zeros(8, dtype=int), np.array([[0, 3]]), False)
    assert np.array_equal(y[0], x[0])
    c, s = np.cos(1.5), np.sin(1.5)
    assert np.allclose([y[1, 0, 0], y[1, 0, 8], y[1, 0, 1], y[1, 0, 63]], [c - 2 * s, 2 * c + s, 3.0, 5.0])
    y = rope.qk_norm_rope(x, None, 0.0, freq, np.zeros(8, dtype=int), np.array([[0, 3]]), True)
    assert np.allclose([y[1, 0, 0], y[1, 0, 1], y[1, 0, 8]], [c - 3 * s, 3 * c + s, 2.0])


def test_norm():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 128)) * 7
    y = rope.qk_norm_rope(x, np.full(128, 2.0), 0.0, np.ones(8), np.zeros(8, dtype=int), np.zeros((1, 3)), False)
    assert np.allclose((y ** 2).mean(-1), 4.0)
    assert np.allclose(rope.qk_norm_rope(np.zeros((1, 1, 128)), np.ones(128), 1e-6, np.ones(8), np.zeros(8, dtype=int), np.zeros((1, 1)), False), 0.0)


def test_products_depend_on_the_distance_alone():
    """q at position p and k at position p - n: their product is the same for every p, on every axis."""
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((2, 1, 1, 64))
    freq, axis = 10000.0 ** (-np.arange(32) / 32), np.arange(32) % 3
    got = []
    for p in (0, 5, 1000):
        pos = np.array([[p], [2 * p], [7 * p]])
        a = rope.qk_norm_rope(q, None, 0.0, freq, axis, pos + np.array([[3], [9], [-4]]), True)
        b = rope.qk_norm_rope(k, None, 0.0, freq, axis, pos, True)
        got.append((a * b).sum())
    assert np.allclose(got, got[0], atol=1e-9)
