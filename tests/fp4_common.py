"""Shared by the tests of the cache of 4-bit codes."""
import numpy as np
import torch

from oracle import fp4

DEV = "cuda:0"
# bf16 rounds a value by at most 2^-8 of it
STEP = 2.0 ** -8


def dev(x):
    return x.to(DEV) if isinstance(x, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def bf16(rng, *shape, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16)


def f64(t):
    return t.float().numpy().astype(np.float64)


def check(got, ref, spread, label="", scores=1.0):
    """Outputs of attention against the definition's, element by element.  What may differ: the output's own rounding; the weights', which
    moves an output by at most 2^-8 of the mean distance of the values from it (numerator and denominator have the same rounded weights;
    1.02 for what is of second order); and 32-bit sums of the scores and outputs, `scores` being how large scores are: some 200 steps of 2^-24 of
    a score of up to 10 times that, 2^-13, of the same distance and of the values."""
    got = got.float().cpu().numpy().astype(np.float64)
    bound = STEP * np.abs(ref) + (1.02 * STEP + scores * 2.0 ** -13) * spread + 2.0 ** -16 * (np.abs(ref) + spread) + 1e-30
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (label, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], ref[bad][:4], bound[bad][:4])


def cache(rng, lens, hkv, d, extra=0, std=1.0, pages=None):
    """A pool with `lens` tokens per request in codes of N(0, std) values and room for `extra` more each; block table.  Slots that no token has, pages
    that no request has: exponents of 255 and random codes, which must not show."""
    need = [-(-(n + extra) // fp4.P) for n in lens]
    pages = pages or sum(need) + 3
    perm = rng.permutation(pages).astype(np.int32)
    bt = np.full((len(lens), max(1, max(need))), perm[-1], dtype=np.int32)      # (a page that no request has: using such an entry would show)
    pool = rng.integers(0, 256, size=(pages, 2, hkv, fp4.slab_bytes(d)), dtype=np.uint8)
    pool[..., fp4.P * d // 2:] = 255
    at = 0
    for r, n in enumerate(need):
        bt[r, :n] = perm[at:at + n]
        at += n
        for j in range(lens[r]):
            fp4.store(pool, bt[r, j // fp4.P], j % fp4.P, rng.standard_normal((hkv, d)) * std, rng.standard_normal((hkv, d)) * std)
    return pool, bt
