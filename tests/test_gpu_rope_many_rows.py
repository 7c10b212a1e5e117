"""GPU tests of the norm and rotation of more than 64 MB of rows, which are read past the caches: the bits of the same rows in smaller calls, which are not."""
import numpy as np
import pytest
import torch

from paper_2401_11181_amd import tetri
from fp4_common import DEV, bf16, dev

pytestmark = pytest.mark.gpu


def outputs(rows, hq, hkv, d):
    return [torch.full((rows, n, d), 7.0, dtype=torch.bfloat16, device=DEV) for n in (hq, hkv)]


def same(a, b):
    return all(torch.equal(x.view(torch.int16).flatten(), y.view(torch.int16).flatten()) for x, y in zip(a, b))


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("d,rows", [(128, 6554), (64, 13108), (128, 7001), (64, 14003)])
def test_bits_of_smaller_calls(d, rows, adjacent):
    hq, hkv, part = 32, 8, 3000
    assert (hq + hkv) * d * 2 * rows > 64 << 20 > (hq + hkv) * d * 2 * part
    rng = np.random.default_rng(16)
    x = dev(bf16(rng, rows, (hq + 2 * hkv) * d))                     # a fused projection's rows
    q, k = x[:, :hq * d], x[:, hq * d:(hq + hkv) * d]
    w = dev(bf16(rng, d) + 1.0)
    pos = rng.integers(0, 100000, size=(2, rows)).astype(np.int32)
    pairs = d // 4 if adjacent else d // 2
    rope = tetri.Rope((1e6 ** (-np.arange(pairs) / pairs)).astype(np.float32), axis=np.arange(pairs) % 2, num_axes=2, adjacent=adjacent)
    h = tetri.Tetri(hq, hkv, d, 64, 16, 16, 16)
    whole, parts = outputs(rows, hq, hkv, d), outputs(rows, hq, hkv, d)
    d_pos = dev(pos)
    h.tetri_qk_norm_rope(q, x.stride(0), k, x.stride(0), w, None, 1e-6, rope, d_pos, None, None, 0, rows, *whole)
    for at in range(0, rows, part):
        n = min(part, rows - at)
        p = dev(pos[:, at:at + n])
        h.tetri_qk_norm_rope(q[at:], x.stride(0), k[at:], x.stride(0), w, None, 1e-6, rope, p, None, None, 0, n, parts[0][at:], parts[1][at:])
        torch.cuda.synchronize()
    assert same(whole, parts) and not (whole[0] == 7.0).all(dim=-1).any()
    # in place
    q, k = q.contiguous(), k.contiguous()
    h.tetri_qk_norm_rope(q, hq * d, k, hkv * d, w, None, 1e-6, rope, d_pos, None, None, 0, rows, q, k)
    torch.cuda.synchronize()
    assert same((q, k), parts)


@pytest.mark.parametrize("d", [128, 64])
def test_a_chunk_with_padding(d):
    """Positions by the chunk's metadata: the bits of calls with given positions, padding rows as they were."""
    hq, hkv, rows, real = 32, 8, 896000 // d, 800000 // d
    rng = np.random.default_rng(17)
    ends = np.sort(rng.choice(np.arange(1, real), size=29, replace=False))
    cu = np.concatenate([[0], ends, [real]]).astype(np.int32)
    ctx = rng.integers(0, 30000, size=30).astype(np.int32)
    q, k = dev(bf16(rng, real, hq * d)), dev(bf16(rng, real, hkv * d))            # (no padding rows at all)
    h = tetri.Tetri(hq, hkv, d, rows, 16, 16, 30)
    rope = tetri.Rope((1e4 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32))
    got, want = outputs(rows, hq, hkv, d), outputs(rows, hq, hkv, d)
    assert (hq + hkv) * d * 2 * rows > 64 << 20
    h.tetri_qk_norm_rope(q, hq * d, k, hkv * d, None, None, 0.0, rope, None, dev(cu), dev(ctx), 30, rows, *got)
    pos = dev(np.concatenate([ctx[s] + np.arange(cu[s + 1] - cu[s]) for s in range(30)]).astype(np.int32)[None])
    for at in range(0, real, 3000):
        n = min(3000, real - at)
        h.tetri_qk_norm_rope(q[at:], hq * d, k[at:], hkv * d, None, None, 0.0, rope, pos[:, at:at + n].contiguous(), None, None, 0, n, want[0][at:], want[1][at:])
        torch.cuda.synchronize()
    assert same(got, want) and (got[0][real:] == 7.0).all() and (got[1][real:] == 7.0).all()
