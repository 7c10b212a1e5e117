"""Pins of the oracle of the cache of 4-bit codes (format: OCP microscaling MXFP4) against things other than itself: values and roundings
written out by hand, closed forms of the attention, and invariants."""
import numpy as np

from oracle import decode as odecode, fp4


def codes_of(x):
    """Codes and exponent of one block whose first values are x, the others 0."""
    block = np.zeros(32)
    block[:len(x)] = x
    codes, exponents = fp4.quantize(block)
    return [int(c) for c in codes[:len(x)]], int(exponents[0])


def test_hand_written_values():
    assert codes_of([4.0, 0.5, 1.0, 1.5, 2.0, 3.0, 6.0, -6.0, -0.0]) == ([6, 1, 2, 3, 4, 5, 7, 15, 8], 127)
    assert codes_of([1.0, 0.125, -0.25]) == ([6, 1, 10], 125)          # largest 1: the power is 1/4
    assert codes_of([0.0]) == ([0], 0)
    assert fp4.dequantize(np.full(32, 15, dtype=np.uint8), np.array([130], dtype=np.uint8))[0] == -48.0


def test_hand_written_roundings():
    # (the 4 keeps the power at 1)
    assert codes_of([4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]) == ([6, 0, 2, 2, 4, 4, 6, 6], 127)       # ties: the even code
    assert codes_of([4.0, 0.2501, 0.7499, 1.2501, 2.4999, 5.001]) == ([6, 1, 1, 3, 4, 7], 127)
    assert codes_of([7.9, -7.0, 6.5]) == ([7, 15, 7], 127)             # above 6: 6
    assert codes_of([2.0 ** -126, 2.0 ** -133, 2.0 ** -127]) == ([4, 0, 2], 0)       # the power stays at 2^-127


def test_values_that_are_not_finite():
    for bad in (np.nan, np.inf, -np.inf):
        assert codes_of([1.0, bad, -2.0]) == ([0, 0, 0], 255)
    assert np.isnan(fp4.dequantize(np.zeros(32, dtype=np.uint8), np.array([255], dtype=np.uint8))).all()


def test_error_and_round_trip():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((50, 128)) * np.exp(rng.uniform(-8, 8, size=(50, 1)))
    codes, exponents = fp4.quantize(x)
    y = fp4.dequantize(codes, exponents)
    # half a step is a quarter of a value between powers of two, or saturation from 8 to 6; below the smallest one a quarter of the power
    power = np.repeat(2.0 ** (exponents.astype(float) - 127), 32, axis=-1)
    assert (np.abs(x - y) <= np.maximum(np.abs(x) * 0.25, power * 0.25) + 1e-12).all()
    again, e2 = fp4.quantize(y)
    same = np.repeat(e2 == exponents, 32, axis=-1)                     # (a block whose largest value is still in its octave)
    assert same.mean() > 0.8 and np.array_equal(again[same] & 7, codes[same] & 7)


def test_bytes_of_a_slab():
    d = 64
    pool = np.zeros((2, 2, 1, fp4.slab_bytes(d)), dtype=np.uint8)
    k = np.zeros((1, d))
    k[0, :3], k[0, 32:35] = [4.0, -2.0, 0.5], [8.0, 1.0, -1.0]
    fp4.store(pool, 1, 5, k, -k)
    assert list(pool[1, 0, 0, 5 * 32:5 * 32 + 2]) == [6 | 12 << 4, 1] and list(pool[1, 0, 0, 5 * 32 + 16:5 * 32 + 18]) == [6 | 1 << 4, 9]
    assert list(pool[1, 0, 0, 16 * 32 + 10:16 * 32 + 12]) == [127, 128] and pool[0].sum() == 0
    assert np.array_equal(fp4.values(pool, d)[1, 1, 0, 5], -k[0])


def test_attention_against_the_oracle_of_the_decode_iteration():
    rng = np.random.default_rng(6)
    hq, hkv, d, ctx = 4, 2, 64, [0, 1, 37]
    bt = np.array([[3, 0, 0], [5, 0, 0], [1, 4, 2]])
    pool = rng.integers(0, 256, size=(6, 2, hkv, fp4.slab_bytes(d)), dtype=np.uint8)
    pool[..., fp4.P * d // 2:] = rng.integers(124, 128, size=pool[..., fp4.P * d // 2:].shape)
    q, k, v = [rng.standard_normal((3, h, d)) for h in (hq, hkv, hkv)]
    got, spread = fp4.attention(q, k, v, pool, bt, [0, 1, 2, 3], ctx, 0.125)
    assert np.allclose(got, odecode.decode_attn(q, k, v, fp4.values(pool, d), bt, ctx, 0.125), atol=1e-12)
    assert np.array_equal(got[0], np.repeat(v[0], 2, axis=0)) and not spread[0].any()


def test_export_then_import_finds_every_token_elsewhere():
    rng = np.random.default_rng(7)
    hkv, d, n, first = 2, 64, [5, 0, 40], [3, 0, 20]
    cu = np.concatenate([[0], np.cumsum(n)])
    src = rng.standard_normal((8, 2, hkv, fp4.P, d))
    bt, bt2 = np.array([[7, 0, 0, 0], [0, 0, 0, 0], [2, 5, 1, 6]]), np.array([[1, 0, 0, 0], [0, 0, 0, 0], [3, 0, 2, 5]])
    buf = fp4.export(src, bt, cu, first)
    assert len(buf) == 2 * hkv * 45 * (d // 2 + d // 32)
    pool = np.full((6, 2, hkv, fp4.slab_bytes(d)), 7, dtype=np.uint8)
    fp4.import_(buf, pool, bt2, cu, first, d)
    want = np.full(pool.shape, 7, dtype=np.uint8)
    for r in range(3):
        for p in range(first[r], first[r] + n[r]):
            row = src[bt[r][p // 16], :, :, p % 16]
            fp4.store(want, bt2[r][p // 16], p % 16, row[0], row[1])
    assert np.array_equal(pool, want)
