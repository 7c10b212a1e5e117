"""Pins of the eviction oracle (oracle/evict.py): hand-written examples, closed forms, torch's CPU softmax and sort as black boxes."""
import numpy as np
import pytest
import torch

from oracle import evict
import evict_common as ec


def pool_of(keys, values=None, page=2):
    """One request, one kv head, its tokens in pages of two slots in reverse order."""
    n, d = len(keys), len(keys[0])
    pages = -(-n // page) + 1
    pool, table = np.zeros((pages, 2, 1, page, d)), np.arange(pages)[::-1].reshape(1, -1)
    for j in range(n):
        pool[table[0][j // page], 0, 0, j % page] = keys[j]
        pool[table[0][j // page], 1, 0, j % page] = keys[j] if values is None else values[j]
    return pool, table


def test_decode_by_hand():
    """Scores 0, ln 2, ln 5: weights 1/8, 2/8, 5/8 on top of what is there; the new token's is written."""
    pool, table = pool_of([[0.0], [np.log(2.0)]])
    w = np.full((2, 1, 2), 7.0)
    evict.decode_weights(np.ones((1, 1, 1)), np.full((1, 1, 1), np.log(5.0)), pool, w, table, [2], 1.0, 1)
    assert np.allclose(w[table[0][0], 0], [7.125, 7.25]) and np.isclose(w[table[0][1], 0, 0], 0.625) and w[table[0][1], 0, 1] == 7.0
    w = np.full((2, 1, 2), 7.0)
    evict.decode_weights(np.ones((1, 1, 1)), np.full((1, 1, 1), np.log(5.0)), pool, w, table, [2], 1.0, 0)
    assert np.allclose(w[table[0][0], 0], [7.125, 7.25]) and (w[table[0][1], 0] == 7.0).all()


def test_prefill_by_hand():
    """Zero keys: row t spreads its weight evenly over the t + 1 + L tokens it sees, one for each of two query heads."""
    pool, table = pool_of([[0.0]] * 5)
    w = np.full((4, 1, 2), 3.0)
    q, k = np.ones((4, 2, 1)), np.zeros((4, 1, 1))
    evict.prefill_weights(q, k, pool, w, table, [0, 3], [2], 2, 1.0)       # two cached tokens, rows 1 and 2 of three
    want = [3 + 2 / 4 + 2 / 5, 3 + 2 / 4 + 2 / 5, 2 / 4 + 2 / 5, 2 / 4 + 2 / 5, 2 / 5]
    got = [w[table[0][j // 2], 0, j % 2] for j in range(5)]
    assert np.allclose(got, want) and w[table[0][2], 0, 1] == 3.0


@pytest.mark.parametrize("last", [1, 3, 50])
def test_prefill_against_torch(last):
    hq, hkv, d = 6, 2, 8
    segs = [(5, 3), (1, 0), (7, 20)]
    c = ec.Cache([L for _, L in segs], hkv, d, 7, room=[n for n, _ in segs])
    gen = torch.Generator().manual_seed(8)
    cu = np.concatenate([[0], np.cumsum([n for n, _ in segs])])
    q, k = torch.randn((14, hq, d), generator=gen).double(), torch.randn((14, hkv, d), generator=gen).double()
    w = torch.nan_to_num(c.weights).double().numpy()
    want = w.copy()
    evict.prefill_weights(q.numpy(), k.numpy(), c.float_pool(), w, c.bt, cu, c.lens, last, 0.3)
    pool = torch.from_numpy(c.float_pool())
    for s, (n, L) in enumerate(segs):
        pages, places = c.slots(s, L + n)
        for h in range(hq):
            keys = torch.cat([pool[pages[:L], 0, h // 3, places[:L]], k[cu[s]:cu[s + 1], h // 3]])
            scores = (q[cu[s]:cu[s + 1], h] @ keys.T) * 0.3
            scores = scores.masked_fill(torch.arange(L + n)[None] > (L + torch.arange(n))[:, None], float("-inf"))
            given = torch.softmax(scores, 1)[max(0, n - last):].sum(0).numpy()
            if h % 3 == 0:
                want[pages[L:], h // 3, places[L:]] = 0.0
            want[pages, h // 3, places] += given
    assert np.allclose(w, want, rtol=1e-12, atol=1e-15)


def test_every_row_gives_one():
    """What all rows give to all slots: one for each (row, query head)."""
    c = ec.Cache([30, 4], 2, 16, 9, room=6)
    c.weights.zero_()
    w = np.zeros(c.weights.shape)
    rng = np.random.default_rng(1)
    evict.prefill_weights(rng.normal(size=(12, 4, 16)), rng.normal(size=(12, 2, 16)), c.float_pool(), w, c.bt, [0, 6, 12], c.lens, 100, 0.5)
    assert np.isclose(w.sum(), 12 * 4)
    w = np.zeros(c.weights.shape)
    evict.decode_weights(rng.normal(size=(2, 4, 16)), rng.normal(size=(2, 2, 16)), c.float_pool(), w, c.bt, c.lens, 0.5, 1)
    assert np.isclose(w.sum(), 2 * 4)


def test_a_chunk_of_one_token_segments_is_a_decode_iteration():
    c = ec.Cache([33, 5, 0], 2, 16, 10, room=1)
    rng = np.random.default_rng(2)
    q, k = rng.normal(size=(3, 4, 16)), rng.normal(size=(3, 2, 16))
    a, b = (torch.nan_to_num(c.weights).double().numpy() for _ in range(2))
    evict.decode_weights(q, k, c.float_pool(), a, c.bt, c.lens, 0.4, 1)
    evict.prefill_weights(q, k, c.float_pool(), b, c.bt, [0, 1, 2, 3], c.lens, 9, 0.4)
    assert np.allclose(a, b, rtol=1e-13)


def weights_of(values):
    w = np.zeros((-(-len(values) // 4), 1, 4), dtype=np.float32)
    w.reshape(-1)[:len(values)] = values
    return w, np.arange(len(w)).reshape(1, -1)


@pytest.mark.parametrize("values,keep,recent,want", [
    # the three heaviest of the first four stay or come to the front, the last two close up
    ([5, 1, 7, 6, 0, 0], 5, 2, [0, 3, 2, 4, 5]),
    # holes are filled in order: slots 0 and 1 by 3 and 5
    ([0, 1, 9, 8, 1, 7, 2, 2], 4, 1, [3, 5, 2, 7]),
    # equal ones: the lowest slots
    ([1, 1, 1, 1, 1], 3, 0, [0, 1, 2]),
    ([1, 1, 1, 1, 1], 3, 1, [0, 1, 4]),
    # only the newest
    ([9, 9, 9, 1, 1], 2, 2, [3, 4]),
    # NaN goes first, -0 is 0
    ([np.nan, -0.0, 0.0, -1, 3], 3, 1, [2, 1, 4]),
    # within the budget
    ([1, 2, 3], 3, 1, [0, 1, 2]), ([1, 2, 3], 5, 1, [0, 1, 2, -1, -1]), ([], 2, 1, [-1, -1]),
])
def test_select_by_hand(values, keep, recent, want):
    w, table = weights_of(values if values else [0])
    slots, lens = evict.select(w, table, [len(values)], keep, recent)
    assert slots[0, 0].tolist() == want and lens.tolist() == [min(keep, len(values))]


def test_select_keeps_what_a_sort_keeps():
    c = ec.Cache([200, 77, 30], 3, 16, 11)
    keep, recent = 50, 12
    slots, lens = evict.select(c.weights.numpy(), c.bt, c.lens, keep, recent)
    for b, L in enumerate(c.lens):
        pages, places = c.slots(b, L)
        for h in range(3):
            got = slots[b, h, :lens[b]].tolist()
            if L <= keep:
                assert got == list(range(L))
                continue
            order = torch.argsort(c.weights[pages, h, places][:L - recent], descending=True, stable=True)[:keep - recent].tolist()
            assert sorted(got) == sorted(order) + list(range(L - recent, L)) and got[-recent:] == list(range(L - recent, L))
            # as few moves as can be: a slot in front that stays is not touched
            assert all(s == i for i, s in enumerate(got[:-recent]) if i in order)
            assert all(s >= i for i, s in enumerate(got))


def test_compact_moves_what_the_map_says():
    c = ec.Cache([60, 20], 2, 16, 12)
    pool, w = np.arange(c.pages * 2 * 2 * 16 * 16).reshape(c.pages, 2, 2, 16, 16), np.arange(c.pages * 2 * 16).reshape(c.pages, 2, 16)
    slots, _ = evict.select(c.weights.numpy(), c.bt, c.lens, 25, 5)
    new_pool, new_w = pool.copy(), w.copy()
    evict.compact(slots, c.bt, c.lens, 25, new_pool, new_w)
    for b, L in enumerate(c.lens):
        pages, places = c.slots(b, L)
        for h in range(2):
            n = min(25, L)
            old = slots[b, h, :n]
            assert np.array_equal(new_pool[pages[:n], :, h, places[:n]], pool[pages[old], :, h, places[old]])
            assert np.array_equal(new_w[pages[:n], h, places[:n]], w[pages[old], h, places[old]])
            assert np.array_equal(new_w[pages[n:], h, places[n:]], w[pages[n:], h, places[n:]])
