"""The weighing calls at shapes that the host's rules send to each of their kernels (tests/host_evict.cpp asserts that they do), the calls on
another stream, and what a decode iteration with weights has to share with the one without."""
import numpy as np
import pytest
import torch

import evict_common as ec
import gpu_common as gc
from test_gpu_evict import dev, handle, run_decode, run_weigh, workspace

pytestmark = pytest.mark.gpu
DEV = gc.DEV

# segments (rows, cached tokens), query heads, kv heads, last rows
WEIGH = {
    "window": ([(512, 16384)], 32, 8, 32),                        # two wavefronts share keys, 64 parts, 64 keys to a wavefront
    "ragged": ([(90, 3000), (40, 7), (101, 1500), (77, 0), (64, 2111), (80, 600), (60, 1999)], 32, 8, 1000),      # two, 3 parts, 32 keys
    "one": ([(256, 600)], 192, 48, 1000),                         # four, 2 parts, 32 keys
    "one-head": ([(1000, 33)], 48, 48, 1000),                     # the same without heads that share a kv head
    "segs": ([(200, 90), (130, 700), (150, 0)], 96, 24, 1000),    # four, 2 parts, 32 keys, several segments
    "segs-wide": ([(200, 1700), (130, 31), (150, 900)], 192, 48, 1000),      # four, not cut, 64 keys, several segments
    "last": ([(300, 1500)], 192, 48, 130),                        # four, 3 parts, 32 keys
    "two-segs": ([(70, 300), (33, 0), (100, 1200)], 96, 24, 1000),           # two, 2 parts, 32 keys
    "two-g3-wide": ([(100, 2600), (45, 500)], 144, 48, 1000),     # two, 2 parts, 64 keys
    "wide": ([(16, 2600)], 48, 48, 1000),                         # none, 10 parts, 64 keys
}


def weigh(segs, hq, hkv, d, last, fp8, scale, seed):
    """The call twice from the same start (bits have to repeat), against torch in 64 bits on the GPU."""
    rows, lens = [n for n, _ in segs], [L for _, L in segs]
    chunk, g = sum(rows), hq // hkv
    c = ec.Cache(lens, hkv, d, seed, fp8, room=rows)
    gen = torch.Generator().manual_seed(seed + 1)
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    q, k = (torch.randn((chunk, n, d), generator=gen).to(torch.bfloat16).to(DEV) for n in (hq, hkv))
    h = handle(c, hq, chunk, len(segs))
    work = workspace(h.tetri_chunk_prefill_weights_workspace(len(segs), max(lens), last))
    pool, got = dev(c.pool), []
    for _ in range(2):
        w = dev(c.weights.clone())
        work.fill_(0xC3)
        h.tetri_chunk_prefill_weights(q, k, pool, w, dev(c.bt), dev(cu), dev(c.ctx), len(segs), max(lens), last, scale, int(fp8), ec.K_SCALE, work,
                                      work.numel())
        got.append(w)
    torch.cuda.synchronize()
    h.close()
    assert torch.equal(got[0].view(torch.int32), got[1].view(torch.int32))
    values = pool.view(torch.float8_e4m3fn).double() * float(np.float32(ec.K_SCALE)) if fp8 else pool.double()
    start = dev(torch.nan_to_num(c.weights)).double()
    before, want, touched, amp = start.clone(), start.clone(), torch.zeros(start.shape, dtype=torch.bool, device=DEV), 0.0
    for s, (n, L) in enumerate(segs):
        pages, places = (dev(x.astype(np.int64)) for x in c.slots(s, L + n))
        looked = min(n, last)
        t = torch.arange(n - looked, n, device=DEV)
        hidden = torch.arange(L + n, device=DEV)[None] > (L + t)[:, None]
        touched[pages, :, places] = True
        before[pages[L:], :, places[L:]] = want[pages[L:], :, places[L:]] = 0.0
        for kh in range(hkv):
            keys = torch.cat([values[pages[:L], 0, kh, places[:L]], k[cu[s]:cu[s + 1], kh].double()]).T.contiguous()
            for head in range(kh * g, kh * g + g):
                x = q[cu[s + 1] - looked:cu[s + 1], head].double()
                want[pages, kh, places] += torch.softmax((x @ keys * scale).masked_fill_(hidden, float("-inf")), 1).sum(0)
                amp = max(amp, float((x.abs() @ keys.abs()).max()) * abs(scale))
    assert torch.equal(got[0].view(torch.int32)[~touched], dev(c.weights).view(torch.int32)[~touched])
    want, before = want[touched].cpu().numpy(), before[touched].cpu().numpy()
    bound = ec.weight_bound(want - before, before, amp, d)
    off = np.abs(got[0][touched].cpu().double().numpy() - want)
    assert (off <= bound).all(), float((off / bound).max())


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", sorted(WEIGH))
def test_weigh(name, d, fp8):
    segs, hq, hkv, last = WEIGH[name]
    weigh(segs, hq, hkv, d, last, fp8, d ** -0.5, 300 + sorted(WEIGH).index(name))


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_weigh_scales_over_codes(scale):
    run_weigh([(40, 100), (24, 0)], 64, 4, 2, 64, 1000, 320, True, scale=scale)


@pytest.mark.parametrize("name", ["ragged", "segs-wide"])
def test_weigh_negative_scale(name):
    segs, hq, hkv, last = WEIGH[name]
    weigh(segs, hq, hkv, 64, last, True, -0.2, 321)


# contexts whose weights a second launch adds: one key past a step, a step's last key, a step's first
DECODE = [2100, 2079, 2080, 5, 0]


@pytest.mark.parametrize("option", [(), (("decode_ranges", 7),), (("decode_parts", 3),)], ids=["default", "ranges", "parts"])
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("append", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_in_two_launches(d, append, fp8, option):
    run_decode(ec.Cache(DECODE, 2, d, 330, fp8), 8, 330, append, d ** -0.5, option)


@pytest.mark.parametrize("lens", [[90, 45, 260], DECODE], ids=["one-launch", "two"])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_decode_scales_over_codes(scale, lens):
    run_decode(ec.Cache(lens, 2, 64, 331, True), 8, 331, 1, scale)


@pytest.mark.parametrize("option", [None, ("decode_ranges", 7), ("decode_parts", 3)], ids=["default", "ranges", "parts"])
@pytest.mark.parametrize("lens", [[1000], [90, 45, 260, 0, 31, 32], DECODE], ids=["one", "short", "long"])
@pytest.mark.parametrize("fp8", [0, 1])
def test_decode_bits(lens, fp8, option):
    """`out` and the pool have the bits of the iteration without weights, and all of it repeats."""
    c, B = ec.Cache(lens, 2, 128, 332, bool(fp8)), len(lens)
    gen = torch.Generator().manual_seed(333)
    q, k, v = (torch.randn((B, n, 128), generator=gen).to(torch.bfloat16).to(DEV) for n in (8, 2, 2))
    h = handle(c, 8)
    if option:
        h.tetri_set_option(*option)
    bt, ctx, most = dev(c.bt), dev(c.ctx), max(lens)
    work = workspace(h.tetri_decode_attn_weights_workspace(B, most))
    got = []
    for _ in range(3):
        pool, w, out = dev(c.pool.clone()), dev(c.weights.clone()), torch.zeros_like(q)
        work.fill_(0xC3)
        h.tetri_decode_attn_weights(q, k, v, pool, w, bt, ctx, B, most, 0.09, 1, fp8, ec.K_SCALE, ec.V_SCALE, work, work.numel(), out)
        got.append((pool, out, w))
    pool, out = dev(c.pool.clone()), torch.zeros_like(q)
    if fp8:
        h.tetri_decode_attn_fp8(q, k, v, pool, bt, ctx, B, most, 0.09, ec.K_SCALE, ec.V_SCALE, 1, out)
    else:
        h.tetri_decode_attn_append(q, k, v, pool, bt, ctx, B, most, 0.09, out)
    torch.cuda.synchronize()
    h.close()
    for again in got:
        assert torch.equal(again[0].view(torch.uint8), pool.view(torch.uint8))
        assert torch.equal(again[1].view(torch.int16), out.view(torch.int16))
        assert torch.equal(again[2].view(torch.int32), got[0][2].view(torch.int32))


@pytest.mark.parametrize("fp8", [0, 1])
def test_all_calls_on_another_stream(fp8):
    """A run of the four calls, one after the other on a stream that is not the current one: the bits of the current one."""
    hq, hkv, d, B, keep, recent, last = 8, 2, 128, 3, 900, 64, 16
    c = ec.Cache([2100, 300, 1500], hkv, d, 340, bool(fp8), room=40)
    gen = torch.Generator().manual_seed(341)
    rand = lambda *s: torch.randn(s, generator=gen).to(torch.bfloat16).to(DEV)
    q, k, v, cq, ck = rand(B, hq, d), rand(B, hkv, d), rand(B, hkv, d), rand(64, hq, d), rand(64, hkv, d)
    bt, ctx, cu = dev(c.bt), dev(c.ctx), dev(np.array([0, 30, 31, 64], dtype=np.int32))
    h, got = handle(c, hq), []
    size = max(h.tetri_decode_attn_weights_workspace(B, 2100), h.tetri_chunk_prefill_weights_workspace(B, 2100, last))
    stream = torch.cuda.Stream()
    for on in (None, stream):
        pool, w, out = dev(c.pool.clone()), dev(torch.nan_to_num(c.weights)), torch.zeros_like(q)
        slots, lens = torch.zeros((B, hkv, keep), dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
        work = workspace(size)
        stream.wait_stream(torch.cuda.current_stream())
        h.tetri_chunk_prefill_weights(cq, ck, pool, w, bt, cu, ctx, B, 2100, last, 0.09, fp8, ec.K_SCALE, work, size, on)
        h.tetri_decode_attn_weights(q, k, v, pool, w, bt, ctx, B, 2100, 0.09, 1, fp8, ec.K_SCALE, ec.V_SCALE, work, size, out, on)
        h.tetri_kv_select(w, bt, ctx, B, 2100, keep, recent, slots, lens, on)
        h.tetri_kv_compact(slots, bt, ctx, B, keep, recent, pool, w, fp8, on)
        (on or torch.cuda.current_stream()).synchronize()
        got.append([t.clone().contiguous().view(torch.uint8) for t in (pool, w, out, slots, lens)])
    h.close()
    for a, b in zip(*got):
        assert torch.equal(a, b)
