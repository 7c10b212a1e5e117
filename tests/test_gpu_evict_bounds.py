"""Eviction and weights of requests whose length is not what the call was told: longer than max_ctx_len, than the block table, below 0."""
import numpy as np
import pytest
import torch

from oracle import evict
import evict_common as ec
import gpu_common as gc
from test_gpu_evict import dev, handle, workspace

pytestmark = pytest.mark.gpu
DEV = gc.DEV


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("max_ctx,keep,recent", [(60, 50, 10), (60, 50, 0), (60, 50, 50), (60, 59, 40), (60, 60, 10), (60, 80, 10), (60, 80, 80), (0, 50, 10),
                                                 (101, 100, 30), (3000, 2900, 2000)])
def test_choice_and_moves_of_a_longer_request(max_ctx, keep, recent, fp8):
    """Only the first max_ctx_len slots are chosen from, and what is moved is what the map says: new slot i holds what slot slots[i] held."""
    c = ec.Cache([100, 40, 60, 61, 200, 3200], 2, 64, 180, fp8, room=max(1, keep))
    c.weights = torch.nan_to_num(c.weights)
    B, looked = len(c.lens), [min(n, max_ctx) for n in c.lens]
    want_slots, want_lens = evict.select(c.weights.numpy(), c.bt, looked, keep, recent)
    h = handle(c, c.hkv)
    pool, weights, bt, ctx = dev(c.pool.clone()), dev(c.weights.clone()), dev(c.bt), dev(c.ctx)
    slots, lens = torch.full((B, c.hkv, keep), 77, dtype=torch.int32, device=DEV), torch.full((B,), 77, dtype=torch.int32, device=DEV)
    h.tetri_kv_select(weights, bt, ctx, B, max_ctx, keep, recent, slots, lens)
    h.tetri_kv_compact(slots, bt, ctx, B, keep, recent, pool, weights, int(fp8))
    torch.cuda.synchronize()
    h.close()
    assert np.array_equal(slots.cpu().numpy(), want_slots) and lens.tolist() == want_lens.tolist()
    bits = torch.uint8 if fp8 else torch.int16
    want_pool, want_weights = c.pool.view(bits).numpy().copy(), c.weights.view(torch.int32).numpy().copy()
    evict.compact(want_slots, c.bt, looked, keep, want_pool, want_weights)
    compared = np.ones((c.pages, ec.PAGE), dtype=bool)
    for b, L in enumerate(looked):                           # (slots that are given up hold nothing of meaning)
        pages, places = c.slots(b, c.lens[b])
        compared[pages[min(keep, L):], places[min(keep, L):]] = False
    assert np.array_equal(pool.cpu().view(bits).numpy().transpose(0, 3, 1, 2, 4)[compared], want_pool.transpose(0, 3, 1, 2, 4)[compared])
    assert np.array_equal(weights.cpu().view(torch.int32).numpy().transpose(0, 2, 1)[compared], want_weights.transpose(0, 2, 1)[compared])
