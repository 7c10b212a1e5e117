"""GPU tests of the norm and the rotation by position of queries and keys, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import rope as orope
from paper_2401_11181_amd import tetri
from fp4_common import DEV, STEP, bf16, dev, f64

pytestmark = pytest.mark.gpu


def check(got, ref, size, angle=0.0, label=""):
    """size: what |y| is at most in the pair.  One rounding to bf16; in front of it about 30 roundings of 2^-24 of `size` (sum of squares, root, products, cosine
    and sine), and the angle's: 64 bits of the position times 2^-53 are nothing, its part of a turn is a 32-bit number, 2 pi 2^-25 off at most."""
    err = np.abs(got.float().cpu().numpy().astype(np.float64) - ref)
    bound = STEP * np.abs(ref) + 2.0 ** -18 * size + 1e-30
    assert (err <= bound).all(), (label, float((err - bound).max()), np.argwhere(err > bound)[:4].tolist())


def sizes(x, weight, eps, pairs, adjacent):
    y = np.abs(orope.qk_norm_rope(x, weight, eps, [], [], np.zeros((1, len(x))), adjacent))
    a, b = (y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2]) if adjacent else (y[..., :pairs], y[..., pairs:2 * pairs])
    s = np.maximum(a, b)
    out = y.copy()
    if adjacent:
        out[..., 0:2 * pairs:2], out[..., 1:2 * pairs:2] = s, s
    else:
        out[..., :pairs], out[..., pairs:2 * pairs] = s, s
    return out


def run(h, hq, hkv, d, q, qs, k, ks, qw, kw, eps, rope, pos=None, cu=None, ctx=None, segs=0, rows=None, fill=7.0):
    q_out = torch.full((rows, hq, d), fill, dtype=torch.bfloat16, device=DEV)
    k_out = torch.full((rows, hkv, d), fill, dtype=torch.bfloat16, device=DEV)
    h.tetri_qk_norm_rope(q, qs, k, ks, qw, kw, eps, rope, pos, cu, ctx, segs, rows, q_out, k_out)
    torch.cuda.synchronize()
    return q_out, k_out


HEADS = [(4, 4, 64), (6, 2, 64), (40, 40, 128), (32, 8, 128), (3, 1, 128), (32, 1, 128), (1, 1, 64)]


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("adjacent", [False, True])
def test_given_positions(heads, adjacent):
    """Fused and separate rows, one to three axes, all kinds of part that turns, with and without norm, one row to hundreds, positions to 10^6 and below 0."""
    hq, hkv, d = heads
    rng = np.random.default_rng(11)
    h = tetri.Tetri(hq, hkv, d, 64, 16, 16, 16)
    for rows, pairs, axes, norm, fused in ((1, d // 2, 1, "both", True), (7, 8, 3, "none", False), (300, d // 4, 2, "q", True), (65, d // 2, 3, "k", False),
                                           (33, 24, 2, "both", True)):
        eps = 1e-6
        freq = (1e6 ** (-np.arange(pairs) / pairs)).astype(np.float32)
        axis = np.arange(pairs) % axes if pairs % 16 else np.arange(pairs) * axes // pairs
        pos = rng.integers(-5, 1000003, size=(axes, rows)).astype(np.int32)
        rope = tetri.Rope(freq, axis=axis, num_axes=axes, adjacent=adjacent)
        if fused:
            x = bf16(rng, rows, (hq + 2 * hkv) * d)
            q, k = x[:, :hq * d], x[:, hq * d:(hq + hkv) * d]
            dx = dev(x)
            dq, dk = dx[:, :hq * d], dx[:, hq * d:(hq + hkv) * d]
        else:
            q, k = bf16(rng, rows, hq * d), bf16(rng, rows, hkv * d)
            dq, dk = dev(q), dev(k)
        w = [bf16(rng, d) + 1.0, bf16(rng, d)]
        if norm in ("none", "k"):
            w[0] = None
        if norm in ("none", "q"):
            w[1] = None
        got = run(h, hq, hkv, d, dq, dq.stride(0), dk, dk.stride(0), *[None if y is None else dev(y) for y in w], eps, rope, pos=dev(pos), rows=rows)
        for x, n, weight, y in ((q, hq, w[0], got[0]), (k, hkv, w[1], got[1])):
            x = f64(x).reshape(rows, n, d)
            weight = None if weight is None else f64(weight)
            ref = orope.qk_norm_rope(x, weight, eps, freq, axis, pos, adjacent)
            check(y, ref, sizes(x, weight, eps, pairs, adjacent), label=str((rows, pairs, axes, norm)))


@pytest.mark.parametrize("segs", [1, 3, 64, 70, 200])
def test_positions_of_a_chunk(segs):
    """Rows of segments begin at their contexts; rows of no segment stay as they are."""
    hq, hkv, d = 4, 2, 128
    rng = np.random.default_rng(12)
    n = rng.integers(1, 5, size=segs)
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    rows = int(cu[-1]) + 9
    ctx = rng.integers(0, 5000, size=segs).astype(np.int32)
    h = tetri.Tetri(hq, hkv, d, 1024, 16, 16, 256)
    q, k = bf16(rng, rows, hq * d), bf16(rng, rows, hkv * d)
    q[cu[-1]:], k[cu[-1]:] = float("nan"), float("nan")
    freq = (10000.0 ** (-np.arange(64) / 64)).astype(np.float32)
    got = run(h, hq, hkv, d, dev(q), hq * d, dev(k), hkv * d, None, None, 1e-6, tetri.Rope(freq), cu=dev(cu), ctx=dev(ctx), segs=segs, rows=rows)
    real = int(cu[-1])
    pos = np.concatenate([ctx[s] + np.arange(n[s]) for s in range(segs)])[None]
    for x, m, y in ((q, hq, got[0]), (k, hkv, got[1])):
        x = f64(x).reshape(rows, m, d)[:real]
        check(y[:real], orope.qk_norm_rope(x, None, 0.0, freq, np.zeros(64, dtype=int), pos, False), sizes(x, None, 0.0, 64, False))
        assert (y[real:] == 7.0).all()


def test_in_place_and_many_rows():
    """The outputs may be the inputs; thousands of rows, one wavefront each: the same bits as out of place."""
    hq, hkv, d, rows = 8, 2, 64, 5000
    rng = np.random.default_rng(13)
    h = tetri.Tetri(hq, hkv, d, 64, 16, 16, 16)
    rope = tetri.Rope((500000.0 ** (-np.arange(32) / 32)).astype(np.float32))
    q, k, w = dev(bf16(rng, rows, hq * d)), dev(bf16(rng, rows, hkv * d)), dev(bf16(rng, d))
    pos = dev(rng.integers(0, 100000, size=(1, rows)).astype(np.int32))
    a = run(h, hq, hkv, d, q, hq * d, k, hkv * d, w, w, 1e-5, rope, pos=pos, rows=rows)
    h.tetri_qk_norm_rope(q, hq * d, k, hkv * d, w, w, 1e-5, rope, pos, None, None, 0, rows, q, k)
    torch.cuda.synchronize()
    assert torch.equal(a[0].view(rows, -1), q) and torch.equal(a[1].view(rows, -1), k)


def test_values_that_are_not_finite_and_zeros():
    """A head of zeros stays 0; an infinity or NaN stays in its pair without a norm, in its head with one."""
    hq, hkv, d = 2, 1, 128
    h = tetri.Tetri(hq, hkv, d, 64, 16, 16, 16)
    rope = tetri.Rope(np.full(16, 0.3, dtype=np.float32))
    q, k = torch.ones((3, hq * d), dtype=torch.bfloat16), torch.zeros((3, hkv * d), dtype=torch.bfloat16)
    q[0, 5], q[1, d + 100] = float("nan"), float("inf")
    pos, one = dev(np.array([[1, 2, 3]], dtype=np.int32)), dev(torch.ones(d, dtype=torch.bfloat16))
    y, z = run(h, hq, hkv, d, dev(q), hq * d, dev(k), hkv * d, None, None, 1e-6, rope, pos=pos, rows=3)
    bad = ~torch.isfinite(y.cpu())
    want = torch.zeros_like(bad)
    want[0, 0, [5, 21]] = True
    want[1, 1, 100] = True
    assert torch.equal(bad, want) and y[1, 1, 100] == float("inf") and not z.any()
    y, z = run(h, hq, hkv, d, dev(q), hq * d, dev(k), hkv * d, one, one, 1e-6, rope, pos=pos, rows=3)
    bad = torch.isnan(y.cpu())
    assert bad[0, 0].all() and bad[1, 1, 100] and not bad[0, 1].any() and not bad[1, 0].any() and not bad[2].any() and not z.any()


def test_on_another_stream_and_replayed():
    hq, hkv, d, rows = 4, 2, 128, 40
    rng = np.random.default_rng(14)
    h = tetri.Tetri(hq, hkv, d, 64, 16, 16, 16)
    freq = (10000.0 ** (-np.arange(64) / 64)).astype(np.float32)
    rope = tetri.Rope(freq)
    q, k = dev(bf16(rng, rows, hq * d)), dev(bf16(rng, rows, hkv * d))
    pos = dev(np.zeros((1, rows), dtype=np.int32))
    q_out, k_out = torch.zeros((rows, hq, d), dtype=torch.bfloat16, device=DEV), torch.zeros((rows, hkv, d), dtype=torch.bfloat16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.tetri_qk_norm_rope(q, hq * d, k, hkv * d, None, None, 1e-6, rope, pos, None, None, 0, rows, q_out, k_out)
    del rope                                             # (the call has read it)
    for step in range(3):
        p = rng.integers(0, 3000, size=(1, rows)).astype(np.int32)
        pos.copy_(dev(p))
        graph.replay()
        torch.cuda.synchronize()
        x = f64(q.cpu()).reshape(rows, hq, d)
        check(q_out, orope.qk_norm_rope(x, None, 0.0, freq, np.zeros(64, dtype=int), p, False), sizes(x, None, 0.0, 64, False))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = q_out.clone()
    q_out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    h.tetri_qk_norm_rope(q, hq * d, k, hkv * d, None, None, 1e-6, tetri.Rope(freq), pos, None, None, 0, rows, q_out, k_out, side)
    side.synchronize()
    assert torch.equal(a, q_out)


def test_refusals():
    h = tetri.Tetri(4, 2, 128, 64, 16, 16, 4)
    q, k = torch.zeros((8, 512), dtype=torch.bfloat16, device=DEV), torch.zeros((8, 256), dtype=torch.bfloat16, device=DEV)
    pos, cu, ctx = [torch.zeros(16, dtype=torch.int32, device=DEV) for _ in range(3)]
    freq = np.ones(64, dtype=np.float32)
    good = dict(q=q, q_stride=512, k=k, k_stride=256, q_weight=None, k_weight=None, eps=1e-6, rope=tetri.Rope(freq), positions=pos, cu_chunk_q_lens=None,
                ctx_lens=None, num_segs=0, num_rows=8, q_out=torch.zeros_like(q), k_out=torch.zeros_like(k))
    h.tetri_qk_norm_rope(**good)
    inf = freq.copy()
    inf[3] = np.inf
    wrong_axis = tetri.Rope(freq)
    wrong_axis.struct.axis[2] = 1
    wide = torch.zeros((8, 640), dtype=torch.bfloat16, device=DEV)
    wrong = [dict(q=None), dict(k_out=None), dict(q=q.view(-1)[4:]), dict(q_stride=504), dict(q_stride=516), dict(k_stride=0), dict(k_stride=-256), dict(eps=-1.0),
             dict(eps=float("nan")), dict(rope=None), dict(rope=tetri.Rope(freq[:4])), dict(rope=tetri.Rope(freq[:20])), dict(rope=tetri.Rope(inf)),
             dict(rope=wrong_axis), dict(rope=tetri.Rope(freq, num_axes=9)), dict(positions=None), dict(cu_chunk_q_lens=cu), dict(positions=None, cu_chunk_q_lens=cu),
             dict(positions=None, cu_chunk_q_lens=cu, ctx_lens=ctx), dict(positions=None, cu_chunk_q_lens=cu, ctx_lens=ctx, num_segs=5), dict(num_rows=0),
             dict(q_weight=q.view(-1)[1:]), dict(q=wide, q_stride=640, q_out=wide)]
    for x in wrong:
        with pytest.raises(tetri.TetriError) as e:
            h.tetri_qk_norm_rope(**{**good, **x})
        assert e.value.status == tetri.TETRI_ERR_INVALID_ARG, x
    with pytest.raises(tetri.TetriError):
        tetri.Tetri(4, 2, 64, 64, 16, 16, 4).tetri_qk_norm_rope(**{**good, "rope": tetri.Rope(freq)})       # 64 pairs of 64 values
    for bad in (dict(freq=np.ones(65)), dict(freq=freq, axis=[0] * 3), dict(freq=freq, axis=[0] * 63 + [1])):
        with pytest.raises(ValueError):
            tetri.Rope(**bad)
