"""Cache of 4-bit codes (test infrastructure only; plain numpy, written from the OCP microscaling formats: MXFP4, blocks of 32 E2M1
elements, 1 sign, 2 exponent bits with bias 1, 1 mantissa bit, under one E8M0 power of two, 255 of which is NaN).

The paper stores the KV cache in the model's 16-bit type; this is an extension of the same kind as oracle/fp8.py.  The reading taken: the power of
a block is 2^(floor(log2 of its largest magnitude) - 2), at least 2^-127; an element is rounded to the nearest code, ties to the even code, and
saturates at 6; a block with a value that is not finite has the exponent 255 and codes of 0.
A pool is bytes [num_pages, 2, Hkv, 16 * (D / 2 + D / 32)]: 16 rows of D / 2 bytes of codes (the even element in the low half), then 16 rows of
D / 32 exponents.
"""
import numpy as np

P = 16
GROUP = 32
VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])


def slab_bytes(d):
    return P * (d // 2 + d // GROUP)


def quantize(x):
    """Codes (uint8 0..15, [..., D]) and exponents (uint8, [..., D / 32]) of values x.  Searches the table of values."""
    x = np.asarray(x, dtype=np.float64)
    y = x.reshape(x.shape[:-1] + (-1, GROUP))
    top = np.abs(y).max(axis=-1)
    finite = np.isfinite(top)
    with np.errstate(divide="ignore"):
        power = np.where(finite & (top > 0), np.floor(np.log2(np.where(finite & (top > 0), top, 1.0))) - 2, -127)
    power = np.maximum(power, -127)
    z = np.where(finite[..., None], np.abs(y), 0.0) / 2.0 ** power[..., None]
    distance = np.abs(np.minimum(z, 6.0)[..., None] - VALUES[:8])
    # (among equally near codes the even one; consecutive values have consecutive codes)
    best = distance.min(axis=-1, keepdims=True)
    order = np.where(distance == best, np.array([0, 1, 0, 1, 0, 1, 0, 1]), 2)
    code = order.argmin(axis=-1)
    code = np.where(finite[..., None], code + 8 * np.signbit(y), 0)
    return code.reshape(x.shape).astype(np.uint8), np.where(finite, power + 127, 255).astype(np.uint8)


def dequantize(codes, exponents):
    """Values (float64) of codes [..., D] and exponents [..., D / 32]."""
    scale = np.where(exponents == 255, np.nan, 2.0 ** (exponents.astype(np.float64) - 127))
    return VALUES[codes] * np.repeat(scale, GROUP, axis=-1)


def pack(codes):
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(raw):
    out = np.empty(raw.shape[:-1] + (2 * raw.shape[-1],), dtype=np.uint8)
    out[..., 0::2], out[..., 1::2] = raw & 15, raw >> 4
    return out


def split(pool, d):
    """Views of a pool: bytes of codes [pages, 2, Hkv, 16, D / 2] and exponents [pages, 2, Hkv, 16, D / 32]."""
    n = P * d // 2
    return pool[..., :n].reshape(pool.shape[:-1] + (P, d // 2)), pool[..., n:].reshape(pool.shape[:-1] + (P, d // GROUP))


def values(pool, d):
    """What a pool holds, [pages, 2, Hkv, 16, D] (float64; NaN under an exponent of 255)."""
    raw, exponents = split(pool, d)
    return dequantize(unpack(raw), exponents)


def store(pool, page, slot, k, v):
    """Rows k, v [Hkv, D] of one token go to a slot (in place)."""
    d = k.shape[-1]
    for which, x in enumerate((k, v)):
        codes, exponents = quantize(x)
        raw = pack(codes)
        for h in range(len(x)):
            pool[page, which, h, slot * d // 2:(slot + 1) * d // 2] = raw[h]
            at = P * d // 2 + slot * (d // GROUP)
            pool[page, which, h, at:at + d // GROUP] = exponents[h]


def append(k_new, v_new, pool, block_table, cu, ctx):
    """A chunk's rows go to the cache (in place): row t of segment s to slot (ctx + t) % 16 of page block_table[s][(ctx + t) / 16]."""
    for s in range(len(ctx)):
        for t in range(int(cu[s + 1]) - int(cu[s])):
            pos = int(ctx[s]) + t
            store(pool, int(block_table[s][pos // P]), pos % P, k_new[int(cu[s]) + t], v_new[int(cu[s]) + t])


def _attend(q, keys, vals, seen, scale):
    """Softmax attention of rows q [n, D] that see the first `seen` keys each, in 64 bits: outputs, and for every output the mean distance of
    the values from it under the weights (what rounding the weights can move it by, per unit of rounding)."""
    s = scale * (q @ keys.T)
    s[np.arange(len(keys))[None] >= np.asarray(seen)[:, None]] = -np.inf
    w = np.exp(s - s.max(axis=1, keepdims=True))
    w /= w.sum(axis=1, keepdims=True)
    out = w @ vals
    spread = np.stack([w[i] @ np.abs(vals - out[i]) for i in range(len(q))])
    return out, spread


def attention(q, k_new, v_new, pool, block_table, cu, ctx, scale):
    """Causal attention of a chunk's segments (a decode iteration: segments of one row) over a pool of codes and their own unquantised rows.
    q [C, Hq, D]; k_new, v_new [C, Hkv, D].  Returns out and spread [C, Hq, D] (zero in rows of no segment)."""
    q, k_new, v_new = [np.asarray(x, dtype=np.float64) for x in (q, k_new, v_new)]
    C, hq, d = q.shape
    hkv = k_new.shape[1]
    g = hq // hkv
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    for s in range(len(ctx)):
        a, b, L = int(cu[s]), int(cu[s + 1]), int(ctx[s])
        pages = np.asarray(block_table[s][:-(-L // P)], dtype=np.int64)
        old = values(pool[pages], d)
        for kh in range(hkv):
            keys = np.concatenate([old[:, 0, kh].reshape(-1, d)[:L], k_new[a:b, kh]])
            vals = np.concatenate([old[:, 1, kh].reshape(-1, d)[:L], v_new[a:b, kh]])
            for h in range(kh * g, (kh + 1) * g):
                out[a:b, h], spread[a:b, h] = _attend(q[a:b, h], keys, vals, L + 1 + np.arange(b - a), scale)
    return out, spread


def export(kv_pages, block_table, cu_tokens, first_tokens=None):
    """Tokens [first_r, first_r + n_r) of every request out of a 16-bit pool [num_pages, 2, Hkv, 16, D] (given as values) as bytes: per
    request codes [2][Hkv][n_r][D / 2], then exponents [2][Hkv][n_r][D / 32]."""
    out = []
    for r in range(len(cu_tokens) - 1):
        n, first = int(cu_tokens[r + 1]) - int(cu_tokens[r]), 0 if first_tokens is None else int(first_tokens[r])
        if n == 0:
            continue
        rows = np.stack([kv_pages[int(block_table[r][p // P]), :, :, p % P] for p in range(first, first + n)], axis=2)
        codes, exponents = quantize(rows)
        out += [pack(codes).reshape(-1), exponents.reshape(-1)]
    return np.concatenate(out) if out else np.zeros(0, dtype=np.uint8)


def import_(buf, pool, block_table, cu_tokens, first_tokens, d):
    """The inverse on the receiver: a buffer's bytes go to the slots of a pool of codes (in place)."""
    hkv = pool.shape[2]
    raw, exponents = [x.copy() for x in split(pool, d)]
    at = 0
    for r in range(len(cu_tokens) - 1):
        n, first = int(cu_tokens[r + 1]) - int(cu_tokens[r]), 0 if first_tokens is None else int(first_tokens[r])
        codes = buf[at:at + 2 * hkv * n * d // 2].reshape(2, hkv, n, d // 2)
        at += codes.size
        exps = buf[at:at + 2 * hkv * n * d // GROUP].reshape(2, hkv, n, d // GROUP)
        at += exps.size
        for t in range(n):
            page, slot = int(block_table[r][(first + t) // P]), (first + t) % P
            raw[page, :, :, slot], exponents[page, :, :, slot] = codes[:, :, t], exps[:, :, t]
    pool[..., :P * d // 2] = raw.reshape(raw.shape[:3] + (-1,))
    pool[..., P * d // 2:] = exponents.reshape(exponents.shape[:3] + (-1,))
