"""GPU parity of the eviction calls (through the C ABI) against the numpy oracle, and a run of them together.

Maps, lengths, and what is moved have to be equal bit for bit.  Weights are fp32: their tolerance counts the roundings
(evict_common.weight_bound).  Outputs of the decode iteration as elsewhere: max-abs 2e-2, mean-abs 2e-3, relative L2 1e-2.
"""
import numpy as np
import pytest
import torch

from oracle import decode as odecode
from oracle import evict
from paper_2401_11181_amd import tetri
from paper_2401_11181_amd.prefill import ChunkedPrefill
import evict_common as ec
import gpu_common as gc

pytestmark = pytest.mark.gpu
DEV = gc.DEV


def handle(c, hq, chunk=64, segs=None):
    return tetri.Tetri(hq, c.hkv, c.d, chunk, c.pages, c.blocks, segs or min(chunk, 8))


def dev(x):
    return (torch.from_numpy(x) if isinstance(x, np.ndarray) else x).to(DEV)


def workspace(n):
    return torch.full((max(n, 16),), 0xC3, dtype=torch.uint8, device=DEV)


def check_weights(c, got, want, before, bound, touched):
    """`touched` [pages, hkv, 16]: slots that the call writes; all others keep their bits."""
    got = got.cpu()
    same = got.view(torch.int32).numpy() == c.weights.view(torch.int32).numpy()
    assert same[~touched].all(), "a weight was written that is none of the call's"
    g, w = got.double().numpy()[touched], want[touched]
    assert np.isfinite(g).all()
    off = np.abs(g - w) - bound[touched]
    assert (off <= 0).all(), ("worst", float((np.abs(g - w) / bound[touched]).max()))


# ---------------------------------------------------------------- decode

DECODE = {
    "mha": ([0, 1, 15, 16, 31, 32, 33, 127, 130, 500], 2, 2, 128),
    "gqa4": ([150, 39, 257], 8, 2, 128),
    "gqa3-d64": ([150, 0, 64, 31], 6, 2, 64),
    "gqa32": ([200, 76], 32, 1, 128),
    "mha-d64": ([97, 0, 63, 2000], 3, 3, 64),
}


def run_decode(c, hq, seed, append, scale, options=(), max_ctx=None, std=1.0):
    gen = torch.Generator().manual_seed(seed + 1)
    B = len(c.lens)
    q = (torch.randn((B, hq, c.d), generator=gen) * std).to(torch.bfloat16)
    k = (torch.randn((B, c.hkv, c.d), generator=gen) * std).to(torch.bfloat16)
    v = torch.randn((B, c.hkv, c.d), generator=gen).to(torch.bfloat16)
    h = handle(c, hq)
    for key, value in options:
        h.tetri_set_option(key, value)
    max_ctx = max(c.lens) if max_ctx is None else max_ctx
    pool, weights = dev(c.pool.clone()), dev(c.weights.clone())
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    work = workspace(h.tetri_decode_attn_weights_workspace(B, max_ctx))
    args = (dev(q), dev(k), dev(v), pool, weights, dev(c.bt), dev(c.ctx), B, max_ctx, scale, append, int(c.fp8), ec.K_SCALE, ec.V_SCALE)
    h.tetri_decode_attn_weights(*args, work, work.numel(), out)
    torch.cuda.synchronize()
    # the same iteration without weights: the pool it leaves
    plain_pool, plain_out = dev(c.pool.clone()), torch.zeros_like(out)
    plain = (args[0], args[1], args[2], plain_pool, args[5], args[6], B, max_ctx, scale)
    if c.fp8:
        h.tetri_decode_attn_fp8(*plain, ec.K_SCALE, ec.V_SCALE, append, plain_out)
    elif append:
        h.tetri_decode_attn_append(*plain, plain_out)
    else:
        h.tetri_decode_attn(*plain, plain_out)
    torch.cuda.synchronize()
    assert torch.equal(pool.view(torch.uint8), plain_pool.view(torch.uint8))
    h.close()
    # the oracle, its amplitude and the slots it writes
    fpool, want = c.float_pool(), torch.nan_to_num(c.weights).double().numpy()
    before = want.copy()
    touched = np.zeros(want.shape, dtype=bool)
    amp = 0.0
    qf, kf = q.double().numpy(), k.double().numpy()
    for b, L in enumerate(c.lens):
        pages, places = c.slots(b, L + append)
        touched[pages, :, places] = True
        if append:
            before[pages[L], :, places[L]] = 0.0
        for kh in range(c.hkv):
            keys = np.concatenate([fpool[pages[:L], 0, kh, places[:L]], kf[b, kh][None]])
            g = hq // c.hkv
            amp = max(amp, ec.amplitude(qf[b, kh * g:kh * g + g], keys, scale))
    evict.decode_weights(qf, kf, fpool, want, c.bt, c.lens, scale, append)
    check_weights(c, weights, want, before, ec.weight_bound(want - before, before, amp, c.d), touched)
    ref = odecode.decode_attn(qf, kf, v.double().numpy(), fpool, c.bt, c.lens, scale)
    gc.compare([out.cpu()], [ref], label="decode with weights")
    return out.cpu(), weights.cpu()


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("append", [0, 1])
@pytest.mark.parametrize("name", sorted(DECODE))
def test_decode(name, append, fp8):
    lens, hq, hkv, d = DECODE[name]
    seed = 40 + sorted(DECODE).index(name)
    run_decode(ec.Cache(lens, hkv, d, seed, fp8), hq, seed, append, d ** -0.5)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("option", [("decode_parts", 1), ("decode_parts", 3), ("decode_parts", 9), ("decode_ranges", 2), ("decode_ranges", 7)],
                         ids=lambda x: "%s-%d" % x)
def test_decode_divisions(option, fp8):
    c = ec.Cache([1, 40, 700, 33, 0, 1500], 2, 128, 60, fp8)
    a = run_decode(c, 8, 60, 1, 128 ** -0.5, [option])
    b = run_decode(c, 8, 60, 1, 128 ** -0.5, [option], max_ctx=c.blocks * 16 - 1)
    assert torch.equal(a[1].nan_to_num(), b[1].nan_to_num()) or option[0] == "decode_ranges"


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_decode_scales(scale):
    run_decode(ec.Cache([90, 45, 260], 2, 64, 61), 4, 61, 1, scale)


def test_decode_long():
    """Contexts of many tiles, some of them one token past a tile."""
    run_decode(ec.Cache([8192, 8193, 5000], 1, 128, 62), 4, 62, 1, 128 ** -0.5)


def test_decode_longer_than_said():
    """Of a request that is longer than max_ctx_len no weight is added; the others' are."""
    c = ec.Cache([100, 30], 2, 128, 63)
    h = handle(c, 4)
    q, k = torch.randn(2, 4, 128, device=DEV).to(torch.bfloat16), torch.randn(2, 2, 128, device=DEV).to(torch.bfloat16)
    w, out = dev(c.weights.clone()), torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=DEV)
    work = workspace(h.tetri_decode_attn_weights_workspace(2, 31))
    h.tetri_decode_attn_weights(q, k, k, dev(c.pool), w, dev(c.bt), dev(c.ctx), 2, 31, 0.1, 0, 0, 1.0, 1.0, work, work.numel(), out)
    w, before = w.cpu(), c.weights
    p, s = c.slots(0, 100)
    assert torch.equal(w[p, :, s], before[p, :, s])
    p, s = c.slots(1, 30)
    assert (w[p, :, s] > before[p, :, s]).all()
    h.close()


def test_decode_longer_than_said_with_append():
    """A request that fills its block table has no slot for a new token: neither its weights nor any other's are touched for it."""
    c = ec.Cache([80, 30], 2, 128, 64, room=[0, 50], extra_blocks=0)
    h = handle(c, 4)
    assert c.blocks == 5
    bf = lambda n: torch.randn(2, n, 128, device=DEV).to(torch.bfloat16)
    w, out = dev(c.weights.clone()), torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=DEV)
    work = workspace(h.tetri_decode_attn_weights_workspace(2, 64))
    h.tetri_decode_attn_weights(bf(4), bf(2), bf(2), dev(c.pool), w, dev(c.bt), dev(c.ctx), 2, 64, 0.1, 1, 0, 1.0, 1.0, work, work.numel(), out)
    w, touched = w.cpu(), torch.zeros(c.weights.shape, dtype=torch.bool)
    p, s = c.slots(1, 31)
    touched[p, :, s] = True
    assert torch.equal(w.view(torch.int32)[~touched], c.weights.view(torch.int32)[~touched])
    assert (w[p, :, s][:30] > c.weights[p, :, s][:30]).all()
    h.close()


@pytest.mark.parametrize("max_ctx,others", [(61, 1), (8193, 1), (1000, 300)])
@pytest.mark.parametrize("append", [0, 1])
def test_decode_a_little_longer_than_said(max_ctx, others, append):
    """One token too many is too many: no weight of that request is added; the longest that are allowed get theirs."""
    lens = [max_ctx + 1] + [max_ctx] + [5] * (others - 1)
    c = ec.Cache(lens, 2, 64, 65, room=[1] * len(lens))
    h = handle(c, 4)
    bf = lambda n: torch.randn(len(lens), n, 64, device=DEV).to(torch.bfloat16)
    w, out = dev(c.weights.clone()), torch.zeros(len(lens), 4, 64, dtype=torch.bfloat16, device=DEV)
    work = workspace(h.tetri_decode_attn_weights_workspace(len(lens), max_ctx))
    h.tetri_decode_attn_weights(bf(4), bf(2), bf(2), dev(c.pool), w, dev(c.bt), dev(c.ctx), len(lens), max_ctx, 0.1, append, 0, 1.0, 1.0, work,
                                work.numel(), out)
    w = w.cpu()
    p, s = c.slots(0, max_ctx + 1 + append)
    assert torch.equal(w[p, :, s].view(torch.int32), c.weights[p, :, s].view(torch.int32))
    for b in range(1, len(lens)):
        p, s = c.slots(b, lens[b])
        assert (w[p, :, s] != c.weights[p, :, s]).float().mean() > 0.9
    h.close()


# ---------------------------------------------------------------- prefill

# segments (rows, cached tokens), chunk, query heads, kv heads, head dim
WEIGH = {
    "one": ([(1, 0)], 64, 2, 2, 128),
    "first-chunk": ([(64, 0)], 64, 4, 2, 64),
    "aligned": ([(64, 128)], 64, 2, 2, 128),
    "ragged": ([(5, 33), (40, 0), (1, 700), (30, 15), (17, 16)], 100, 6, 2, 128),
    "gqa8": ([(100, 300), (28, 1)], 128, 8, 1, 64),
    "gqa32": ([(9, 40)], 16, 32, 1, 128),
    "gqa5": ([(33, 70), (20, 0)], 64, 10, 2, 64),
    "gqa40": ([(21, 50)], 32, 40, 1, 64),
    "long": ([(200, 2500), (56, 130)], 300, 4, 4, 128),
}


def run_weigh(segs, chunk, hq, hkv, d, last, seed, fp8, scale=None, std=1.0, slack=0):
    rows, lens = [n for n, _ in segs], [L for _, L in segs]
    c = ec.Cache(lens, hkv, d, seed, fp8, room=rows, std=std, extra_blocks=2 + -(-slack // ec.PAGE))
    gen = torch.Generator().manual_seed(seed + 1)
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    q = (torch.randn((chunk, hq, d), generator=gen) * std).to(torch.bfloat16)
    k = (torch.randn((chunk, hkv, d), generator=gen) * std).to(torch.bfloat16)
    q[cu[-1]:], k[cu[-1]:] = float("nan"), float("nan")      # padding rows are never read
    scale = d ** -0.5 if scale is None else scale
    h = handle(c, hq, chunk, min(chunk, len(segs) + slack))
    weights = dev(c.weights.clone())
    max_ctx = max(lens) + slack
    work = workspace(h.tetri_chunk_prefill_weights_workspace(len(segs), max_ctx, last))
    args = (dev(q), dev(k), dev(c.pool), weights, dev(c.bt), dev(cu), dev(c.ctx), len(segs), max_ctx, last, scale, int(fp8), ec.K_SCALE,
            work, work.numel())
    h.tetri_chunk_prefill_weights(*args)
    torch.cuda.synchronize()
    h.close()
    fpool, want = c.float_pool(), torch.nan_to_num(c.weights).double().numpy()
    before, touched, amp = want.copy(), np.zeros(want.shape, dtype=bool), 0.0
    qf, kf = torch.nan_to_num(q).double().numpy(), torch.nan_to_num(k).double().numpy()
    g = hq // hkv
    for s, (n, L) in enumerate(segs):
        pages, places = c.slots(s, L + n)
        touched[pages, :, places] = True
        before[pages[L:], :, places[L:]] = 0.0
        for kh in range(hkv):
            keys = np.concatenate([fpool[pages[:L], 0, kh, places[:L]], kf[cu[s]:cu[s + 1], kh]])
            amp = max(amp, ec.amplitude(qf[cu[s + 1] - min(n, last):cu[s + 1], kh * g:kh * g + g].reshape(-1, d), keys, scale))
    evict.prefill_weights(qf, kf, fpool, want, c.bt, cu, lens, last, scale)
    check_weights(c, weights, want, before, ec.weight_bound(want - before, before, amp, d), touched)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("last", [1, 7, 32, 1000])
@pytest.mark.parametrize("name", sorted(WEIGH))
def test_weigh(name, last, fp8):
    run_weigh(*WEIGH[name], last, 80 + sorted(WEIGH).index(name), fp8)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_weigh_scales(scale):
    run_weigh([(40, 100), (24, 0)], 64, 4, 2, 64, 1000, 95, False, scale=scale)


def test_weigh_bounds_that_are_not_reached():
    """max_ctx_len above the longest context, room for more segments than there are."""
    run_weigh([(40, 100), (24, 0), (30, 333)], 100, 4, 2, 128, 1000, 96, False, slack=700)


def test_weigh_many_segments():
    """More segments than lanes of a wavefront."""
    run_weigh([(1 + i % 3, (37 * i) % 90) for i in range(90)], 200, 2, 1, 64, 2, 97, False)


@pytest.mark.parametrize("hq,hkv,d,n,L,last,fp8", [
    (32, 16, 64, 300, 8000, 300, False),          # hundreds of rows a kv head, 64 keys to a wavefront
    (16, 16, 128, 700, 7700, 700, True),
    (8, 2, 128, 40, 9000, 16, False),             # few rows, keys in many parts
    (4, 4, 128, 513, 0, 2000, False),             # no context
])
def test_weigh_large(hq, hkv, d, n, L, last, fp8):
    """Against torch in 64 bits, on the GPU."""
    c = ec.Cache([L], hkv, d, 99, fp8, room=n)
    gen = torch.Generator().manual_seed(100)
    q, k = (torch.randn((n, heads, d), generator=gen).to(torch.bfloat16).to(DEV) for heads in (hq, hkv))
    h = handle(c, hq, n, 1)
    weights = dev(torch.nan_to_num(c.weights))
    want = weights.double()
    work = workspace(h.tetri_chunk_prefill_weights_workspace(1, L, last))
    h.tetri_chunk_prefill_weights(q, k, dev(c.pool), weights, dev(c.bt), dev(np.array([0, n], dtype=np.int32)), dev(c.ctx), 1, L, last, d ** -0.5,
                                  int(fp8), ec.K_SCALE, work, work.numel())
    pages, places = (dev(x.astype(np.int64)) for x in c.slots(0, L + n))
    pool = torch.from_numpy(c.float_pool()).to(DEV)
    rows = min(n, last)
    t = torch.arange(n - rows, n, device=DEV)
    hidden = torch.arange(L + n, device=DEV)[None] > (L + t)[:, None]
    want[pages[L:], :, places[L:]] = 0.0
    before, amp = want.clone(), 0.0
    for kh in range(hkv):
        keys = torch.cat([pool[pages[:L], 0, kh, places[:L]], k[:, kh].double()])
        for head in range(kh * hq // hkv, (kh + 1) * hq // hkv):
            x = q[n - rows:, head].double()
            want[pages, kh, places] += torch.softmax((x @ keys.T * d ** -0.5).masked_fill(hidden, float("-inf")), 1).sum(0)
            amp = max(amp, float((x.abs() @ keys.abs().T).max()) * d ** -0.5)
    want, before = want.cpu().numpy(), before.cpu().numpy()
    bound = ec.weight_bound(want - before, before, amp, d)
    off = np.abs(weights.cpu().double().numpy() - want)
    assert (off <= bound).all(), float((off / bound).max())
    h.close()


def test_weigh_scores_far_above_the_first_ones():
    """Two keys score 127.5 (as a power of two) above those before them: exp2 of that is finite, of twice it is not."""
    c = ec.Cache([100], 1, 64, 101, room=1)
    h = handle(c, 1, 8, 1)
    c.pool.zero_()
    pages, places = c.slots(0, 101)
    for j in (64, 68):                           # (in different halves of a wavefront)
        c.pool[pages[j], 0, 0, places[j], 0] = 8.0
    q, k = torch.zeros((8, 1, 64), dtype=torch.bfloat16), torch.zeros((8, 1, 64), dtype=torch.bfloat16)
    q[0, 0, 0] = 8.0
    w = dev(torch.zeros_like(c.weights))
    work = workspace(h.tetri_chunk_prefill_weights_workspace(1, 100, 1))
    h.tetri_chunk_prefill_weights(dev(q), dev(k), dev(c.pool), w, dev(c.bt), dev(np.array([0, 1], dtype=np.int32)), dev(c.ctx), 1, 100, 1,
                                  127.5 / 64 / 1.4426950408889634, 0, 1.0, work, work.numel())
    got = w.cpu()[pages, 0, places]
    want = torch.zeros(101)
    want[[64, 68]] = 0.5
    assert torch.allclose(got, want, rtol=0, atol=1e-5)
    h.close()


def test_weigh_large_scores():
    """Scores of some hundreds: one key takes nearly all of a row's weight, and the largest lies anywhere."""
    run_weigh([(64, 400)], 64, 2, 2, 128, 1000, 98, False, std=6.0)


# ---------------------------------------------------------------- select

def run_select(c, keep, recent, max_ctx=None, pad=0):
    h = handle(c, c.hkv)
    B = len(c.lens)
    slots = torch.full((B, c.hkv, keep), 77, dtype=torch.int32, device=DEV)
    lens = torch.full((B,), 77, dtype=torch.int32, device=DEV)
    w = dev(c.weights)
    h.tetri_kv_select(w, dev(c.bt), dev(c.ctx), B, max_ctx or max(c.lens) + pad, keep, recent, slots, lens)
    torch.cuda.synchronize()
    assert torch.equal(w.cpu().view(torch.int32), c.weights.view(torch.int32))
    h.close()
    want, want_lens = evict.select(c.weights.numpy(), c.bt, c.lens, keep, recent)
    assert np.array_equal(lens.cpu().numpy(), want_lens)
    assert np.array_equal(slots.cpu().numpy(), want)
    return slots.cpu(), lens.cpu()


def fill_weights(c, kind, seed):
    gen = torch.Generator().manual_seed(seed)
    w = torch.randn(c.weights.shape, generator=gen)
    if kind == "spread":
        w = (w * 6).exp()
    elif kind == "few":                          # many equal ones
        w = torch.randint(0, 3, w.shape, generator=gen).float()
    elif kind == "zero":
        w = torch.where(w > 0, 0.0, -0.0)
    elif kind == "close":                        # that differ in their last bits only
        w = (torch.randint(0, 64, w.shape, generator=gen) + 0x3F000000).to(torch.int32).view(torch.float32)
    elif kind == "odd":                          # negative ones, infinities, NaN, subnormal ones
        w[torch.rand(w.shape, generator=gen) < 0.2] = float("nan")
        w[torch.rand(w.shape, generator=gen) < 0.1] = float("inf")
        w[torch.rand(w.shape, generator=gen) < 0.2] = float("-inf")
        w[torch.rand(w.shape, generator=gen) < 0.1] = 1e-42
    c.weights = w.contiguous()


@pytest.mark.parametrize("keep,recent", [(1, 0), (1, 1), (50, 0), (50, 16), (50, 50), (300, 31), (555, 100), (4000, 5)])
@pytest.mark.parametrize("kind", ["spread", "few", "zero", "close", "odd"])
def test_select(kind, keep, recent):
    c = ec.Cache([0, 1, 49, 50, 51, 52, 64, 300, 556, 1000], 2, 64, 120, room=max(1, keep))
    fill_weights(c, kind, 121)
    run_select(c, keep, recent, pad=(keep * 7) % 50)


@pytest.mark.parametrize("length", [2048, 2049, 4097, 8193, 16384, 16385, 32768, 32769, 40000])
def test_select_long(length):
    c = ec.Cache([length, 9], 1, 64, 122)
    for kind in ("spread", "few"):
        fill_weights(c, kind, 123)
        run_select(c, length // 3, 100)


@pytest.mark.parametrize("kind", ["spread", "few", "zero", "close", "odd", "fourth", "rising", "wide"])
@pytest.mark.parametrize("length", [8200, 12288, 16384, 20001, 32768])
def test_select_long_kinds(length, kind):
    """Weights of which some, by their place, say something else than all do."""
    c = ec.Cache([length, 9], 1, 64, 126)
    if kind in ("fourth", "rising", "wide"):
        j = torch.arange(16 * c.blocks, dtype=torch.float32)
        gen = torch.Generator().manual_seed(127)
        w = {"fourth": torch.where(j % 4 == 0, 2.0, 1e-3) * (1 + torch.rand(j.shape, generator=gen)), "rising": j / 1000 - 3,
             "wide": torch.exp2(200 * torch.rand(j.shape, generator=gen) - 100) * torch.where(torch.rand(j.shape, generator=gen) < 0.3, -1.0, 1.0)}[kind]
        pages, places = c.slots(0, length)
        c.weights[pages, 0, places] = w[:length]
    else:
        fill_weights(c, kind, 128)
    for keep, recent in ((1, 0), (101, 3), (length // 8, 256), (length // 4, 0), (length // 2, 0), (length - 1, 7)):
        run_select(c, keep, recent)


def test_select_under_the_largest_bound():
    c = ec.Cache([1000, 70], 1, 64, 124, extra_blocks=(1 << 19) // 16)
    fill_weights(c, "spread", 125)
    run_select(c, 300, 20, max_ctx=1 << 19)


# ---------------------------------------------------------------- compact

COMPACT = [(1, 0), (1, 1), (50, 0), (50, 16), (50, 50), (280, 31), (555, 100), (600, 600), (4000, 5)]


def run_compact(c, keep, recent):
    slots, _ = evict.select(c.weights.numpy(), c.bt, c.lens, keep, recent)
    h = handle(c, c.hkv)
    pool, weights = dev(c.pool.clone()), dev(c.weights.clone())
    h.tetri_kv_compact(dev(slots), dev(c.bt), dev(c.ctx), len(c.lens), keep, recent, pool, weights, int(c.fp8))
    torch.cuda.synchronize()
    h.close()
    bits = torch.uint8 if c.fp8 else torch.int16
    want_pool, want_weights = c.pool.view(bits).numpy().copy(), c.weights.view(torch.int32).numpy().copy()
    evict.compact(slots, c.bt, c.lens, keep, want_pool, want_weights)
    got_pool, got_weights = pool.cpu().view(bits).numpy(), weights.cpu().view(torch.int32).numpy()
    compared = np.ones((c.pages, ec.PAGE), dtype=bool)       # (slots that are given up hold nothing of meaning)
    for b, L in enumerate(c.lens):
        pages, places = c.slots(b, L)
        compared[pages[keep:], places[keep:]] = False
    assert np.array_equal(got_pool.transpose(0, 3, 1, 2, 4)[compared], want_pool.transpose(0, 3, 1, 2, 4)[compared])
    assert np.array_equal(got_weights.transpose(0, 2, 1)[compared], want_weights.transpose(0, 2, 1)[compared])
    return slots, pool, weights


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("keep,recent", COMPACT)
def test_compact(keep, recent, d, fp8):
    c = ec.Cache([0, 1, 49, 50, 51, 52, 64, 300, 556, 1000], 2, d, 140, fp8, room=max(1, keep))
    run_compact(c, keep, recent)


@pytest.mark.parametrize("length,keep,recent", [(5000, 4999, 4999), (5000, 4990, 3000), (5000, 2500, 2500), (5000, 3900, 2100), (3300, 1500, 1025)])
def test_compact_many_recent(length, keep, recent):
    """More recent tokens than the workgroup that moves them has places for at a time; they overlap where they go to."""
    run_compact(ec.Cache([length, 700], 1, 64, 141), keep, recent)


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_prefill_decode_evict_decode(fp8):
    """Chunks are prefilled, cached and weighed, tokens decoded, the cache cut, tokens decoded again, cut again: outputs and
    the weights follow the oracle over the tokens that are left."""
    hq, hkv, d, chunk, scale = 4, 2, 64, 48, 64 ** -0.5
    lens, keep, recent = [130, 60, 45], 64, 10
    c = ec.Cache([0, 0, 0], hkv, d, 160, fp8, room=[n + 30 for n in lens])
    B = len(lens)
    h = handle(c, hq, chunk, 4)
    gen = torch.Generator().manual_seed(161)
    pool, weights, bt = dev(c.pool.clone()), dev(c.weights.clone()), dev(c.bt)
    ref_w = torch.nan_to_num(c.weights).double().numpy()
    work = workspace(max(h.tetri_chunk_prefill_weights_workspace(3, max(lens), 1000), h.tetri_decode_attn_weights_workspace(B, 190)))
    have = [0, 0, 0]

    def float_pool():
        c.pool = pool.cpu()
        return c.float_pool()

    while have != lens:                          # chunk by chunk, all requests together
        rows = [min(16, lens[b] - have[b]) for b in range(B)]
        live = [b for b in range(B) if rows[b]]
        cu = np.concatenate([[0], np.cumsum([rows[b] for b in live])]).astype(np.int32)
        q = torch.randn((chunk, hq, d), generator=gen).to(torch.bfloat16)
        k, v = (torch.randn((chunk, hkv, d), generator=gen).to(torch.bfloat16) for _ in range(2))
        table, ctx = c.bt[live], np.array([have[b] for b in live], dtype=np.int32)
        evict.prefill_weights(q.double().numpy(), k.double().numpy(), float_pool(), ref_w, table, cu, ctx, 1000, scale)
        args = (dev(q), dev(k), dev(v), pool, dev(table), dev(cu), dev(ctx), len(live), scale)
        out = torch.zeros((chunk, hq, d), dtype=torch.bfloat16, device=DEV)
        h.tetri_chunk_prefill_weights(args[0], args[1], pool, weights, args[4], args[5], args[6], len(live), int(ctx.max()), 1000, scale,
                                      int(fp8), ec.K_SCALE, work, work.numel())
        if fp8:
            h.tetri_chunk_prefill_attn_fp8(*args, ec.K_SCALE, ec.V_SCALE, 1, out)
        else:
            h.tetri_chunk_prefill_attn_append(*args, out)
        have = [have[b] + rows[b] for b in range(B)]
    for turn in range(2):
        for _ in range(9):
            q = torch.randn((B, hq, d), generator=gen).to(torch.bfloat16)
            k, v = (torch.randn((B, hkv, d), generator=gen).to(torch.bfloat16) for _ in range(2))
            before = float_pool()
            evict.decode_weights(q.double().numpy(), k.double().numpy(), before, ref_w, c.bt, have, scale, 1)
            ref = odecode.decode_attn(q.double().numpy(), k.double().numpy(), v.double().numpy(), before, c.bt, have, scale)
            out = torch.zeros((B, hq, d), dtype=torch.bfloat16, device=DEV)
            h.tetri_decode_attn_weights(dev(q), dev(k), dev(v), pool, weights, bt, dev(np.array(have, dtype=np.int32)), B, max(have), scale, 1,
                                        int(fp8), ec.K_SCALE, ec.V_SCALE, work, work.numel(), out)
            gc.compare([out.cpu()], [ref], label="turn %d" % turn)
            have = [n + 1 for n in have]
        got = weights.cpu().double().numpy()
        for b in range(B):
            pages, places = c.slots(b, have[b])
            # (d + ... roundings a term, see evict_common; some hundred terms, all positive)
            assert np.allclose(got[pages, :, places], ref_w[pages, :, places], rtol=1e-4, atol=1e-7)
        # the choice goes by the weights as the library has them
        ref_w = np.nan_to_num(got)
        c.weights = weights.cpu()
        slots, new_lens = evict.select(c.weights.numpy(), c.bt, have, keep, recent)
        d_slots, d_lens = torch.zeros((B, hkv, keep), dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
        d_ctx = dev(np.array(have, dtype=np.int32))
        h.tetri_kv_select(weights, bt, d_ctx, B, max(have), keep, recent, d_slots, d_lens)
        assert np.array_equal(d_slots.cpu().numpy(), slots) and d_lens.tolist() == new_lens.tolist()
        want_pool = pool.cpu().view(torch.uint8 if fp8 else torch.int16).numpy().copy()
        evict.compact(slots, c.bt, have, keep, want_pool, ref_w)
        h.tetri_kv_compact(d_slots, bt, d_ctx, B, keep, recent, pool, weights, int(fp8))
        have = [int(n) for n in new_lens]
        got_pool = pool.cpu().view(torch.uint8 if fp8 else torch.int16).numpy()
        for b in range(B):
            pages, places = c.slots(b, have[b])
            assert np.array_equal(got_pool[pages, :, :, places], want_pool[pages, :, :, places])
        assert have == [64, 64, 54] if turn == 0 else have == [64, 64, 63]
    h.close()


def test_weights_of_a_scheduled_batch():
    """ChunkedPrefill.weights: every chunk of a packed batch, against the oracle over the same chunks."""
    hq, hkv, d, C, scale = 4, 2, 64, 48, 0.125
    prompts = [70, 33, 90]
    c = ec.Cache([0, 0, 0], hkv, d, 175, room=prompts, extra_blocks=0)
    sess = ChunkedPrefill(prompts, None, C, hq, hkv, d, c.pages, [list(c.bt[b, :-(-n // 16)]) for b, n in enumerate(prompts)])
    gen = torch.Generator().manual_seed(176)
    bf = lambda n: [torch.randn((m, n, d), generator=gen).to(torch.bfloat16) for m in prompts]
    q, k, v = bf(hq), bf(hkv), bf(hkv)
    pool, w = dev(c.pool), dev(torch.nan_to_num(c.weights))
    want = torch.nan_to_num(c.weights).double().numpy()
    for chunk in range(sess.n_chunks):
        cq, ck, cv = (sess.gather_chunk([dev(t) for t in x], chunk) for x in (q, k, v))
        segs = sess.chunk_segments(chunk)
        cu = np.concatenate([[0], np.cumsum([n for _, _, n in segs])])
        c.pool = pool.cpu()
        evict.prefill_weights(cq.cpu().double().numpy(), ck.cpu().double().numpy(), c.float_pool(), want, c.bt[[r for r, _, _ in segs]], cu,
                              [start for _, start, _ in segs], 16, scale)
        work = workspace(sess.weights_workspace(chunk, 16))
        sess.weights(chunk, cq, ck, pool, w, scale, 16, work)
        sess.append(chunk, ck, cv, pool)
    got = w.cpu().double().numpy()
    for b, n in enumerate(prompts):
        pages, places = c.slots(b, n)
        # (some hundred terms, all positive; 64 products a score: see evict_common)
        assert np.allclose(got[pages, :, places], want[pages, :, places], rtol=1e-4, atol=1e-7)


def test_captured_and_replayed():
    """All four calls in a graph, replayed with eager work in between: every replay adds what an eager call adds."""
    hq, hkv, d = 4, 2, 128
    c = ec.Cache([300, 77], hkv, d, 170, room=20)
    h = handle(c, hq, 32, 4)
    B, keep, recent = 2, 100, 16
    bf = lambda *s: torch.randn(s, device=DEV).to(torch.bfloat16)
    q, k, v, cq, ck = bf(B, hq, d), bf(B, hkv, d), bf(B, hkv, d), bf(32, hq, d), bf(32, hkv, d)
    cu, bt, ctx = dev(np.array([0, 17, 31], dtype=np.int32)), dev(c.bt), dev(c.ctx)
    start_pool, start_w = dev(c.pool), dev(torch.nan_to_num(c.weights))
    pool, w = start_pool.clone(), start_w.clone()
    work = [workspace(h.tetri_decode_attn_weights_workspace(B, 300)), workspace(h.tetri_chunk_prefill_weights_workspace(2, 300, 8))]
    out, slots, lens = torch.zeros_like(q), torch.zeros((B, hkv, keep), dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)

    def calls():
        h.tetri_chunk_prefill_weights(cq, ck, pool, w, bt, cu, ctx, B, 300, 8, 0.09, 0, 1.0, work[1], work[1].numel())
        h.tetri_decode_attn_weights(q, k, v, pool, w, bt, ctx, B, 300, 0.09, 1, 0, 1.0, 1.0, work[0], work[0].numel(), out)
        h.tetri_kv_select(w, bt, ctx, B, 300, keep, recent, slots, lens)
        h.tetri_kv_compact(slots, bt, ctx, B, keep, recent, pool, w, 0)

    def reset():
        pool.copy_(start_pool)
        w.copy_(start_w)
        for t in (out, slots, lens):
            t.zero_()

    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in (pool, w, out, slots, lens)]
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(4):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((pool, w, out, slots, lens), want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        reset()
        calls()                                  # eager, between the replays
        torch.cuda.synchronize()
        assert torch.equal(w.view(torch.uint8), want[1].view(torch.uint8))
    h.close()


def test_far_pages():
    """Pages behind more than 4 GB of pool and of codes, and what the same request gives in a small pool."""
    hq, hkv, d, keep, recent = 16, 8, 128, 40, 10
    c = ec.Cache([90], hkv, d, 173, room=1)
    got = []
    for pages in (c.pages, 140000):
        bt = np.where(c.bt < c.pages, c.bt + pages - c.pages, c.bt)
        h = tetri.Tetri(hq, hkv, d, 64, pages, c.blocks, 8)
        pool, w = torch.empty((pages, 2, hkv, 16, d), dtype=torch.bfloat16, device=DEV), torch.empty((pages, hkv, 16), device=DEV)
        pool[pages - c.pages:], w[pages - c.pages:] = dev(c.pool), dev(c.weights)
        gen = torch.Generator().manual_seed(174)
        q, k, v = (torch.randn((1, n, d), generator=gen).to(torch.bfloat16).to(DEV) for n in (hq, hkv, hkv))
        work = workspace(max(h.tetri_decode_attn_weights_workspace(1, 90), h.tetri_chunk_prefill_weights_workspace(1, 90, 1)))
        out, slots = torch.zeros_like(q), torch.zeros((1, hkv, keep), dtype=torch.int32, device=DEV)
        lens, ctx, table = torch.zeros(1, dtype=torch.int32, device=DEV), dev(c.ctx), dev(bt)
        cq, ck = torch.zeros((64, hq, d), dtype=torch.bfloat16, device=DEV), torch.zeros((64, hkv, d), dtype=torch.bfloat16, device=DEV)
        cq[:1], ck[:1] = q, k
        h.tetri_chunk_prefill_weights(cq, ck, pool, w, table, dev(np.array([0, 1], dtype=np.int32)), ctx, 1, 90, 1, 0.09, 0, 1.0, work, work.numel())
        h.tetri_decode_attn_weights(q, k, v, pool, w, table, ctx, 1, 90, 0.09, 1, 0, 1.0, 1.0, work, work.numel(), out)
        h.tetri_kv_select(w, table, ctx, 1, 90, keep, recent, slots, lens)
        h.tetri_kv_compact(slots, table, ctx, 1, keep, recent, pool, w, 0)
        used = slice(pages - c.pages, pages)
        got.append([x.cpu() for x in (pool[used], w[used], out, slots, lens)])
        h.close()
    for a, b in zip(*got):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_another_stream():
    c = ec.Cache([400, 30], 2, 64, 171)
    h = handle(c, 2)
    stream = torch.cuda.Stream()
    slots, lens = torch.zeros((2, 2, 50), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    w, bt, ctx = dev(c.weights), dev(c.bt), dev(c.ctx)
    stream.wait_stream(torch.cuda.current_stream())
    h.tetri_kv_select(w, bt, ctx, 2, 400, 50, 5, slots, lens, stream)
    stream.synchronize()
    want, _ = evict.select(c.weights.numpy(), c.bt, c.lens, 50, 5)
    assert np.array_equal(slots.cpu().numpy(), want)
    h.close()


def test_refusals():
    """Nothing is launched: the pointers behind these calls are never followed.  (All refusals, without a GPU: test_host_evict.py.)"""
    c = ec.Cache([20], 2, 64, 172)
    h = handle(c, 4)
    x, i = torch.zeros(4096, dtype=torch.bfloat16, device=DEV), torch.zeros(64, dtype=torch.int32, device=DEV)
    f = torch.zeros(64, device=DEV)
    for call in (lambda: h.tetri_decode_attn_weights(x, x, x, x, f, i, i, 1, 20, 0.1, 1, 0, 1.0, 1.0, x, 16, x),
                 lambda: h.tetri_chunk_prefill_weights(x, x, x, f, i, i, i, 1, 20, 0, 0.1, 0, 1.0, x, 1 << 20),
                 lambda: h.tetri_kv_select(f, i, i, 1, 20, 4, 5, i, x),
                 lambda: h.tetri_kv_select(f, i, i, 1, 20, 4, 2, i, i),
                 lambda: h.tetri_kv_compact(i, i, i, 0, 4, 2, x, f, 0)):
        with pytest.raises(tetri.TetriError) as e:
            call()
        assert e.value.status == tetri.TETRI_ERR_INVALID_ARG
    h.close()
