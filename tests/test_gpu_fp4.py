"""GPU tests of the cache of 4-bit codes: export, import and the decode iteration, against the oracle (oracle/fp4.py): bytes bit for bit, outputs to
bounds that follow from what is rounded."""
import numpy as np
import pytest
import torch

from oracle import fp4
from paper_2401_11181_amd import tetri
from fp4_common import DEV, bf16, cache, check, dev, f64

pytestmark = pytest.mark.gpu
P = fp4.P


# ---------------------------------------------------------------- export and import

def handle(hq, hkv, d, pages, blocks, chunk=64, segs=8):
    return tetri.Tetri(hq, hkv, d, chunk, pages, blocks, segs)


def test_quantiser_on_every_bf16_value_under_every_power():
    """Every bf16 bit pattern in blocks whose largest value has each exponent, so that each value meets each power it can: two values of a block are the
    largest one's, the others are 30 patterns that are no larger (and patterns that are not finite, in blocks of their own)."""
    rng = np.random.default_rng(91)
    blocks = []
    for field in list(range(0, 12)) + list(range(100, 140)) + list(range(250, 255)):
        for low in (0, 8, 20, 40, 127):                              # patterns down from the block's largest one
            top = field << 7 | rng.integers(0, 128)
            most = top + 1
            body = (top - rng.integers(0, min(most, 128 * 7 + low), size=30)) if low else rng.integers(0, most, size=30)
            blocks.append(np.concatenate([[top, top | 0x8000], np.maximum(body, 0) | rng.integers(0, 2, size=30) << 15]))
    for bits in np.arange(0, 65536).reshape(-1, 32):                 # every pattern, with its neighbours
        blocks.append(bits)
    for bad in (0x7F80, 0xFF80, 0x7FC0, 0x7F81):
        blocks.append(np.concatenate([[bad], rng.integers(0, 0x7F80, size=31)]))
    hkv, d = 2, 128
    while (len(blocks) * 32) % (2 * hkv * P * d):
        blocks.append(np.zeros(32, dtype=np.int64))
    pool = np.array(blocks).astype(np.uint16).reshape(-1, 2, hkv, P, d)
    pages = len(pool)
    n = pages * P
    bt = rng.permutation(pages).astype(np.int32)[None]
    cu = np.array([0, n], dtype=np.int32)
    buf = torch.zeros(2 * hkv * n * (d // 2 + d // 32), dtype=torch.uint8, device=DEV)
    h = handle(hkv, hkv, d, pages, pages)
    h.tetri_kv_export_fp4(dev(pool.view(np.int16)), dev(bt), dev(cu), None, 1, n, buf)
    with np.errstate(invalid="ignore"):
        want = fp4.export((pool.astype(np.uint32) << 16).view(np.float32), bt, cu)
    got = buf.cpu().numpy()
    bad = np.nonzero(got != want)[0]
    assert bad.size == 0, (bad.size, bad[:5], got[bad[:5]], want[bad[:5]])


MOVES = {"one": ([1], [0], 4, 128), "ragged": ([5, 0, 33, 16, 1, 100], [3, 7, 15, 0, 31, 2], 2, 128), "ragged-d64": ([40, 1, 0, 17, 250], None, 3, 64),
         "many": ([1] * 100 + [0] * 30 + [2] * 7, None, 1, 64), "long": ([700, 300], [1, 900], 5, 128)}


@pytest.mark.parametrize("slabs", [0, 1, 3])
@pytest.mark.parametrize("name", sorted(MOVES))
def test_export_and_import(name, slabs):
    n, first, hkv, d = MOVES[name]
    rng = np.random.default_rng(92)
    R = len(n)
    reach = [a + (first[r] if first else 0) for r, a in enumerate(n)]
    need = [-(-x // P) for x in reach]
    pages, blocks = sum(need) + 2, max(1, max(need))

    def table():
        bt, perm, at = np.zeros((R, blocks), dtype=np.int32), rng.permutation(pages), 0
        for r in range(R):
            bt[r, :need[r]] = perm[at:at + need[r]]
            at += need[r]
        return bt
    bt, bt2 = table(), table()
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    total = int(cu[-1])
    f = None if first is None else np.array(first, dtype=np.int32)
    pool = bf16(rng, pages, 2, hkv, P, d)
    h = handle(hkv, hkv, d, pages, blocks)
    if slabs:
        h.tetri_set_option("transfer_slabs", slabs)
    size = 2 * hkv * total * (d // 2 + d // 32)
    guarded = torch.full((size + 64,), 170, dtype=torch.uint8, device=DEV)
    f_dev = None if f is None else dev(f)
    h.tetri_kv_export_fp4(dev(pool), dev(bt), dev(cu), f_dev, R, total, guarded)
    want = fp4.export(f64(pool), bt, cu, f)
    got = guarded.cpu().numpy()
    assert np.array_equal(got[:size], want) and (got[size:] == 170).all()
    # what arrives is any bytes
    data = rng.integers(0, 256, size=size, dtype=np.uint8)
    codes = rng.integers(0, 256, size=(pages, 2, hkv, fp4.slab_bytes(d)), dtype=np.uint8)
    d_codes = dev(codes)
    h.tetri_kv_import_fp4(dev(data), dev(bt2), dev(cu), f_dev, R, total, d_codes)
    fp4.import_(data, codes, bt2, cu, f, d)
    assert np.array_equal(d_codes.cpu().numpy(), codes)


def test_moving_nothing():
    h = handle(2, 2, 64, 4, 4)
    cu = dev(np.zeros(3, dtype=np.int32))
    bt = dev(np.zeros((2, 4), dtype=np.int32))
    pool = torch.zeros((4, 2, 2, fp4.slab_bytes(64)), dtype=torch.uint8, device=DEV)
    h.tetri_kv_import_fp4(None, bt, cu, None, 2, 0, pool)
    h.tetri_kv_export_fp4(torch.zeros((4, 2, 2, P, 64), dtype=torch.bfloat16, device=DEV), bt, cu, None, 2, 0, None)
    assert not pool.any()


# ---------------------------------------------------------------- decode

def run_decode(q, k, v, pool, bt, ctx, scale, append=0, options=(), blocks=None, max_ctx=None, h=None):
    B, hq, d = q.shape
    h = h or tetri.Tetri(hq, k.shape[1], d, 64, len(pool), blocks or bt.shape[1], 8)
    for key, value in options:
        h.tetri_set_option(key, value)
    d_pool = dev(pool)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    h.tetri_decode_attn_fp4(dev(q), dev(k), dev(v), d_pool, dev(bt), dev(np.array(ctx, dtype=np.int32)), B, max(ctx) if max_ctx is None else max_ctx, scale,
                            append, out)
    torch.cuda.synchronize()
    return out.cpu(), d_pool.cpu().numpy()


WAYS = {"auto": (), "one-part": (("decode_parts", 1),), "parts3": (("decode_parts", 3),), "parts40": (("decode_parts", 40),), "ranges5": (("decode_ranges", 5),),
        "ranges60": (("decode_ranges", 60),)}
SHAPES = {"mha": (2, 2, 128), "gqa3": (6, 2, 64), "gqa4": (8, 2, 128), "mha-d64": (3, 3, 64), "gqa16": (16, 1, 128), "gqa17": (17, 1, 64), "gqa32": (32, 1, 128),
          "gqa32-d64": (64, 2, 64)}
LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 127, 128, 129, 500]


@pytest.mark.parametrize("way", sorted(WAYS))
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_decode(shape, way):
    """Lengths around every edge of a step, with append (whose bytes are the oracle's, and no others change); then without it, the same bits."""
    hq, hkv, d = SHAPES[shape]
    rng = np.random.default_rng(93)
    pool, bt = cache(rng, LENS, hkv, d, extra=1)
    q, k, v = bf16(rng, len(LENS), hq, d), bf16(rng, len(LENS), hkv, d), bf16(rng, len(LENS), hkv, d)
    ref, spread = fp4.attention(f64(q), f64(k), f64(v), pool, bt, np.arange(len(LENS) + 1), LENS, d ** -0.5)
    out, after = run_decode(q, k, v, pool, bt, LENS, d ** -0.5, 1, WAYS[way])
    check(out, ref, spread, "%s %s" % (shape, way))
    want = pool.copy()
    fp4.append(f64(k), f64(v), want, bt, np.arange(len(LENS) + 1), LENS)
    assert np.array_equal(after, want)
    again, after = run_decode(q, k, v, pool, bt, LENS, d ** -0.5, 0, WAYS[way])
    assert np.array_equal(after, pool) and torch.equal(again.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.7, 30.0])
@pytest.mark.parametrize("way", ["one-part", "ranges5"])
def test_decode_scales(scale, way):
    rng = np.random.default_rng(94)
    lens = [200, 0, 45, 90]
    pool, bt = cache(rng, lens, 2, 128)
    q, k, v = bf16(rng, 4, 4, 128), bf16(rng, 4, 2, 128), bf16(rng, 4, 2, 128)
    ref, spread = fp4.attention(f64(q), f64(k), f64(v), pool, bt, np.arange(5), lens, scale)
    out, _ = run_decode(q, k, v, pool, bt, lens, scale, 0, WAYS[way])
    check(out, ref, spread, str(scale), scores=max(1.0, abs(scale) * 128 ** 0.5))


def test_every_code_under_many_powers():
    """V holds every code under powers from 2^-120 to 2^100 in turn, K zeros: outputs are means of the tokens' values."""
    hq, hkv, d, L = 2, 2, 128, 64
    pool = np.zeros((5, 2, hkv, fp4.slab_bytes(d)), dtype=np.uint8)
    bt = np.array([[2, 0, 4, 1]], dtype=np.int32)
    rng = np.random.default_rng(95)
    for power in (-120, -60, -3, 0, 5, 60, 100):
        pool[:, 1] = rng.integers(0, 256, size=pool[:, 1].shape)
        pool[:, 1, :, P * d // 2:] = 127 + power + rng.integers(0, 3, size=pool[:, 1, :, P * d // 2:].shape)
        q, k, v = bf16(rng, 1, hq, d), bf16(rng, 1, hkv, d) * 0, bf16(rng, 1, hkv, d) * 2.0 ** power
        ref, spread = fp4.attention(f64(q), f64(k), f64(v), pool, bt, [0, 1], [L], 1.0)
        out, _ = run_decode(q, k, v, pool, bt, [L], 1.0)
        check(out, ref, spread, str(power))


def test_powers_of_k_reach_the_scores():
    """K's blocks have powers from 2^-6 to 2^2, another for each group: a group's exponent that met another's codes would show."""
    rng = np.random.default_rng(96)
    for hq, hkv, d in ((4, 2, 128), (3, 3, 64)):
        lens = [100, 37]
        pool, bt = cache(rng, lens, hkv, d)
        at = P * d // 2
        live = pool[:, 0, :, at:] != 255
        pool[:, 0, :, at:][live] = (127 + rng.integers(-6, 3, size=live.sum())).astype(np.uint8)
        q, k, v = bf16(rng, 2, hq, d), bf16(rng, 2, hkv, d), bf16(rng, 2, hkv, d)
        ref, spread = fp4.attention(f64(q), f64(k), f64(v), pool, bt, [0, 1, 2], lens, 0.05)
        out, _ = run_decode(q, k, v, pool, bt, lens, 0.05)
        check(out, ref, spread, str(d), scores=4.0)


def test_not_a_number_stays_where_it_is():
    """A group of V that is NaN makes NaN of its 32 elements of the outputs of its kv head; a key of NaN of the whole head's output; other requests and heads
    have the bits that they have without."""
    rng = np.random.default_rng(97)
    hq, hkv, d, lens = 4, 2, 128, [70, 40]
    pool, bt = cache(rng, lens, hkv, d)
    q, k, v = bf16(rng, 2, hq, d), bf16(rng, 2, hkv, d), bf16(rng, 2, hkv, d)
    good, _ = run_decode(q, k, v, pool, bt, lens, 0.1, 0, WAYS["parts3"])
    for which, slot in ((1, 3), (0, 50)):
        bad = pool.copy()
        bad[bt[0, slot // P], which, 1, P * d // 2 + slot % P * 4 + 2] = 255
        out, _ = run_decode(q, k, v, bad, bt, lens, 0.1, 0, WAYS["parts3"])
        nan = torch.isnan(out)
        want = torch.zeros_like(nan)
        want[0, 2:, 64:96] = True
        if which == 0:
            want[0, 2:] = True
        assert torch.equal(nan, want)
        assert torch.equal(out[~nan], good[~nan])


def test_large_scores_and_rising_ones():
    """Scores that rise from key to key by far more than the exponent's reserve, and infinities of the new token's."""
    rng = np.random.default_rng(98)
    d, L = 64, 200
    pool, bt = cache(rng, [L], 1, d)
    for j in range(L):
        row = np.zeros((1, d))
        row[0, 0] = 0.5 * j
        fp4.store(pool, bt[0, j // P], j % P, row, rng.standard_normal((1, d)))
    q, k, v = torch.zeros((1, 2, d), dtype=torch.bfloat16), bf16(rng, 1, 1, d), bf16(rng, 1, 1, d)
    q[0, 0, 0], q[0, 1, 0] = 4.0, -4.0
    for way in ("one-part", "parts3"):
        ref, spread = fp4.attention(f64(q), f64(k), f64(v), pool, bt, [0, 1], [L], 1.0)
        out, _ = run_decode(q, k, v, pool, bt, [L], 1.0, 0, WAYS[way])
        check(out, ref, spread, way, scores=40.0)


def test_results_do_not_depend_on_the_bound_or_on_what_lies_behind():
    """The same bits with a larger max_ctx_len (one part), and whatever unused slots and block-table entries hold."""
    rng = np.random.default_rng(99)
    lens = [33, 100, 0, 16]
    pool, bt = cache(rng, lens, 2, 128)
    q, k, v = bf16(rng, 4, 4, 128), bf16(rng, 4, 2, 128), bf16(rng, 4, 2, 128)
    a, _ = run_decode(q, k, v, pool, bt, lens, 0.1, 0, WAYS["one-part"])
    b, _ = run_decode(q, k, v, pool, bt, lens, 0.1, 0, WAYS["one-part"], max_ctx=bt.shape[1] * P)
    clean = pool.copy()
    raw_unused = np.ones((len(pool), P), dtype=bool)
    for r, n in enumerate(lens):
        for j in range(n):
            raw_unused[bt[r, j // P], j % P] = False
    for page, slot in np.argwhere(raw_unused):
        fp4.store(clean, page, slot, np.zeros((2, 128)), np.zeros((2, 128)))
    c, _ = run_decode(q, k, v, clean, bt, lens, 0.1, 0, WAYS["one-part"])
    assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(a.view(torch.int16), c.view(torch.int16))


def test_replayed_decode_steps():
    """A captured iteration with append, replayed for three tokens with other inputs in the same buffers and eager calls in between."""
    rng = np.random.default_rng(100)
    hq, hkv, d, lens = 8, 2, 128, [40, 5, 300]
    pool, bt = cache(rng, lens, hkv, d, extra=4)
    h = tetri.Tetri(hq, hkv, d, 64, len(pool), bt.shape[1], 8)
    d_pool, d_bt = dev(pool), dev(bt)
    q, k, v = [torch.zeros((3, n, d), dtype=torch.bfloat16, device=DEV) for n in (hq, hkv, hkv)]
    ctx, out = dev(np.array(lens, dtype=np.int32)), torch.zeros((3, hq, d), dtype=torch.bfloat16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.tetri_decode_attn_fp4(q, k, v, d_pool, d_bt, ctx, 3, 303, 0.1, 1, out)
    d_pool.copy_(dev(pool))
    for step in range(4):
        x = [bf16(rng, 3, n, d) for n in (hq, hkv, hkv)]
        for to, src in zip((q, k, v), x):
            to.copy_(src)
        now = [n + step for n in lens]
        ctx.copy_(dev(np.array(now, dtype=np.int32)))
        if step == 2:
            h.tetri_decode_attn_fp4(q, k, v, d_pool, d_bt, ctx, 3, 303, 0.1, 1, out)
        else:
            graph.replay()
        torch.cuda.synchronize()
        ref, spread = fp4.attention(f64(x[0]), f64(x[1]), f64(x[2]), pool, bt, [0, 1, 2, 3], now, 0.1)
        check(out, ref, spread, "step %d" % step)
        fp4.append(f64(x[1]), f64(x[2]), pool, bt, [0, 1, 2, 3], now)
        assert np.array_equal(d_pool.cpu().numpy(), pool)


def test_refusals():
    h = tetri.Tetri(4, 2, 128, 64, 8, 4, 4)
    q, k = torch.zeros((2, 4, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((2, 2, 128), dtype=torch.bfloat16, device=DEV)
    pool = torch.zeros((8, 2, 2, fp4.slab_bytes(128)), dtype=torch.uint8, device=DEV)
    bt, ctx = torch.zeros((2, 4), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    cu = torch.zeros(3, dtype=torch.int32, device=DEV)
    good = dict(q=q, k_new=k, v_new=k, kv_pages_fp4=pool, block_table=bt, ctx_lens=ctx, num_reqs=2, max_ctx_len=63, scale=0.1, append=1, out=q.clone())
    h.tetri_decode_attn_fp4(**good)
    wrong = [dict(q=None), dict(kv_pages_fp4=pool.view(-1)[8:]), dict(block_table=None), dict(ctx_lens=None), dict(num_reqs=0), dict(max_ctx_len=64),
             dict(max_ctx_len=-1), dict(scale=float("inf")), dict(append=2), dict(append=-1), dict(out=None)]
    for x in wrong:
        with pytest.raises(tetri.TetriError) as e:
            h.tetri_decode_attn_fp4(**{**good, **x})
        assert e.value.status == tetri.TETRI_ERR_INVALID_ARG, x
    with pytest.raises(tetri.TetriError) as e:
        tetri.Tetri(33, 1, 128, 64, 8, 4, 4).tetri_decode_attn_fp4(**good)
    assert e.value.status == tetri.TETRI_ERR_UNSUPPORTED
    rows = torch.zeros((8, 2, 2, P, 128), dtype=torch.bfloat16, device=DEV)
    buf = torch.zeros(1 << 16, dtype=torch.uint8, device=DEV)
    for call in (lambda: h.tetri_kv_export_fp4(None, bt, cu, None, 2, 4, buf), lambda: h.tetri_kv_export_fp4(rows, bt, cu, None, 2, 4, None),
                 lambda: h.tetri_kv_export_fp4(rows, bt, cu, None, 0, 4, buf), lambda: h.tetri_kv_export_fp4(rows, bt, cu, None, 2, 129, buf),
                 lambda: h.tetri_kv_import_fp4(buf[8:], bt, cu, None, 2, 4, pool), lambda: h.tetri_kv_import_fp4(buf, None, cu, None, 2, 4, pool),
                 lambda: h.tetri_kv_import_fp4(buf, bt, cu, None, 2, -1, pool)):
        with pytest.raises(tetri.TetriError) as e:
            call()
        assert e.value.status == tetri.TETRI_ERR_INVALID_ARG
