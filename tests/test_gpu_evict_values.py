"""Weights of a chunk that holds infinities and NaN: they reach the keys that such a row sees, and no others."""
import numpy as np
import pytest
import torch

from oracle import evict
import evict_common as ec
import gpu_common as gc
from test_gpu_evict import dev, handle, workspace

pytestmark = pytest.mark.gpu
DEV = gc.DEV


def run(segs, hq, hkv, d, last, seed, fp8, spoil, scale=None):
    """spoil(q, k, c, cu) puts its values in; the oracle, whose rows see what they see, says where NaN is to be."""
    rows, lens = [n for n, _ in segs], [L for _, L in segs]
    chunk = sum(rows) + 7
    c = ec.Cache(lens, hkv, d, seed, fp8, room=rows)
    gen = torch.Generator().manual_seed(seed + 1)
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    q, k = (torch.randn((chunk, n, d), generator=gen).to(torch.bfloat16) for n in (hq, hkv))
    scale = d ** -0.5 if scale is None else scale
    clean_q, clean_k, clean_pool = q.double().numpy(), k.double().numpy(), c.float_pool()
    bad_pool = spoil(q, k, c, cu)
    h = handle(c, hq, chunk, len(segs))
    weights = dev(c.weights.clone())
    work = workspace(h.tetri_chunk_prefill_weights_workspace(len(segs), max(lens), last))
    h.tetri_chunk_prefill_weights(dev(q), dev(k), dev(c.pool), weights, dev(c.bt), dev(cu), dev(c.ctx), len(segs), max(lens), last, scale, int(fp8),
                                  ec.K_SCALE, work, work.numel())
    torch.cuda.synchronize()
    h.close()
    fpool, want = clean_pool, torch.nan_to_num(c.weights).double().numpy()
    for page, kh, place in bad_pool or ():
        fpool[page, 0, kh, place] = np.nan
    before, touched, amp, g = want.copy(), np.zeros(want.shape, dtype=bool), 0.0, hq // hkv
    for s, (n, L) in enumerate(segs):
        pages, places = c.slots(s, L + n)
        touched[pages, :, places] = True
        before[pages[L:], :, places[L:]] = 0.0
        for kh in range(hkv):
            keys = np.nan_to_num(np.concatenate([fpool[pages[:L], 0, kh, places[:L]], clean_k[cu[s]:cu[s + 1], kh]]))
            amp = max(amp, ec.amplitude(clean_q[cu[s + 1] - min(n, last):cu[s + 1], kh * g:kh * g + g].reshape(-1, d), keys, scale))
    with np.errstate(invalid="ignore"):
        evict.prefill_weights(q.double().numpy(), k.double().numpy(), fpool, want, c.bt, cu, lens, last, scale)
    got = weights.cpu()
    assert (got.view(torch.int32).numpy() == c.weights.view(torch.int32).numpy())[~touched].all()
    got, nan = got.double().numpy(), np.isnan(want)
    assert (touched & nan).any() and (touched & ~nan).any()
    assert np.array_equal(np.isnan(got)[touched], nan[touched])
    fine = touched & ~nan
    bound = ec.weight_bound(want[fine] - before[fine], before[fine], amp, d)
    assert (np.abs(got[fine] - want[fine]) <= bound).all()


# rows (token, query head) of the first segment; a row gives nothing to the chunk's tokens behind it
ROWS = [(0, 0), (5, 1), (31, 0), (32, 3), (40, 2), (63, 1)]


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")], ids=["nan", "inf", "-inf"])
@pytest.mark.parametrize("row", ROWS, ids=lambda x: "%d-%d" % x)
@pytest.mark.parametrize("hq,hkv,d,fp8", [(4, 2, 128, False), (4, 4, 64, True), (4, 1, 64, False)])
def test_query_rows(hq, hkv, d, fp8, row, value):
    def spoil(q, k, c, cu):
        q[row[0], row[1], 3] = value
    run([(100, 40), (30, 0)], hq, hkv, d, 1000, 200, fp8, spoil, scale=-0.1 if row[0] == 31 else None)


@pytest.mark.parametrize("token", [0, 7, 31, 32, 45])
@pytest.mark.parametrize("last", [20, 50])
def test_rows_that_are_looked_at(token, last):
    """A row in front of the last ones is not looked at; a NaN there reaches nothing.  One in another segment makes something to see."""
    def spoil(q, k, c, cu):
        q[token] = float("nan")
        q[cu[1] + 12, 0] = float("nan")
    run([(60, 33), (30, 5)], 2, 2, 64, last, 201, False, spoil)


@pytest.mark.parametrize("hq,hkv,d,fp8", [(16, 16, 64, False), (16, 16, 128, True)])
def test_query_rows_of_wide_workgroups(hq, hkv, d, fp8):
    """64 keys to a wavefront."""
    def spoil(q, k, c, cu):
        q[3, 2, 0], q[33, 5], q[34, 5, 1] = float("nan"), float("inf"), float("-inf")
    run([(70, 8000)], hq, hkv, d, 1000, 202, fp8, spoil)


def test_row_whose_scores_are_all_minus_infinity():
    def spoil(q, k, c, cu):
        k[:, :, 0] = 1.0
        q[9], q[9, 0, 0] = 0.0, float("-inf")
    run([(50, 0), (20, 0)], 1, 1, 64, 1000, 203, False, spoil)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_cached_key(fp8):
    """It makes NaN of its request and kv head, and of nothing else."""
    def spoil(q, k, c, cu):
        pages, places = c.slots(0, 41)
        c.pool[pages[40], 0, 1, places[40], 5] = ec.NAN_CODE if fp8 else float("nan")
        return [(pages[40], 1, places[40])]
    run([(60, 90), (30, 70)], 4, 2, 64, 1000, 204, fp8, spoil)


def test_new_key():
    def spoil(q, k, c, cu):
        k[17, 0, 5] = float("nan")
    run([(60, 90), (30, 70)], 4, 2, 128, 1000, 205, False, spoil)


def test_workgroups_that_go_over_many_segments():
    """More tiles of keys than workgroups abreast: what one segment's rows leave behind is none of the next one's."""
    segs = [(20 + i % 5, 3 * i) for i in range(30)]

    def spoil(q, k, c, cu):
        for s in range(0, 30, 3):
            q[cu[s] + s % 20, s::7, 1] = float("nan")
    run(segs, 64, 64, 64, 1000, 206, False, spoil)
