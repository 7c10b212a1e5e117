"""Oracle of eviction from the paged KV cache by accumulated attention weight (test infrastructure only; plain numpy, float64).

An extension of this build, not of the paper: TetriInfer Sec. 3.4 names the memory of the decode instance as what limits its
batch.  Beside the pool one number per (page, kv head, slot) is kept: how much softmax weight the token there has received.
kv_weights [num_pages, Hkv, P] is updated in place, everything else is returned.
"""
import math

import numpy as np


def _softmax(s):
    w = np.exp(s - s.max())
    return w / w.sum()


def _key_row(kv_pages, table, j):
    P = kv_pages.shape[3]
    return kv_pages[int(table[j // P]), 0, :, j % P, :]


def prefill_weights(q, k_new, kv_pages, kv_weights, block_table, cu, ctx_lens, last_rows, scale):
    """Adds what the last rows of every segment give: q [C,Hq,D], k_new [C,Hkv,D], kv_pages [num_pages,2,Hkv,P,D]."""
    Hq, Hkv, P = q.shape[1], k_new.shape[1], kv_pages.shape[3]
    g = Hq // Hkv
    for s in range(len(ctx_lens)):
        L, first, n = int(ctx_lens[s]), int(cu[s]), int(cu[s + 1] - cu[s])
        keys = np.zeros((L + n, Hkv, q.shape[2]))
        for j in range(L + n):
            keys[j] = _key_row(kv_pages, block_table[s], j) if j < L else k_new[first + j - L]
        given = np.zeros((L + n, Hkv))
        for t in range(max(0, n - last_rows), n):
            for h in range(Hq):
                seen = L + t + 1
                given[:seen, h // g] += _softmax(scale * (keys[:seen, h // g] @ q[first + t, h].astype(np.float64)))
        for j in range(L + n):
            page, slot = int(block_table[s][j // P]), j % P
            kv_weights[page, :, slot] = given[j] + (kv_weights[page, :, slot] if j < L else 0.0)


def decode_weights(q, k_new, kv_pages, kv_weights, block_table, ctx_lens, scale, append):
    """Adds what a decode iteration gives: q [B,Hq,D], k_new [B,Hkv,D]."""
    B, Hq, D = q.shape
    Hkv, P = k_new.shape[1], kv_pages.shape[3]
    g = Hq // Hkv
    for b in range(B):
        L = int(ctx_lens[b])
        keys = np.zeros((L + 1, Hkv, D))
        for j in range(L):
            keys[j] = _key_row(kv_pages, block_table[b], j)
        keys[L] = k_new[b]
        for h in range(Hkv):
            given = sum(_softmax(scale * (keys[:, h] @ q[b, h * g + i].astype(np.float64))) for i in range(g))
            for j in range(L):
                kv_weights[int(block_table[b][j // P]), h, j % P] += given[j]
            if append:
                kv_weights[int(block_table[b][L // P]), h, L % P] = given[L]


def select(kv_weights, block_table, ctx_lens, keep, recent):
    """Returns (slots [B,Hkv,keep] int32, new_lens [B] int32)."""
    _, Hkv, P = kv_weights.shape
    B = len(ctx_lens)
    slots = np.full((B, Hkv, keep), -1, dtype=np.int32)
    new_lens = np.zeros(B, dtype=np.int32)
    for b in range(B):
        L = int(ctx_lens[b])
        n = min(L, keep)
        r = min(recent, n)
        new_lens[b] = n
        for h in range(Hkv):
            if L <= keep:
                slots[b, h, :L] = range(L)
                continue
            weight = [float(kv_weights[int(block_table[b][j // P]), h, j % P]) for j in range(L - r)]
            weight = [-math.inf if math.isnan(w) else w for w in weight]
            stays = set(sorted(range(L - r), key=lambda j: (-weight[j], j))[:n - r])
            moving = iter(sorted(j for j in stays if j >= n - r))
            for i in range(n):
                slots[b, h, i] = i + L - n if i >= n - r else (i if i in stays else next(moving))
    return slots, new_lens


def compact(slots, block_table, ctx_lens, keep, kv_pages, kv_weights):
    """Moves tokens of the pool [num_pages,2,Hkv,P,D] and their weights, in place: new slot i holds what slot slots[b][h][i] held."""
    P = kv_pages.shape[3]
    old_pages, old_weights = kv_pages.copy(), kv_weights.copy()
    for b in range(len(ctx_lens)):
        for h in range(kv_pages.shape[2]):
            for i in range(min(int(ctx_lens[b]), keep)):
                j = int(slots[b, h, i])
                to, frm = int(block_table[b][i // P]), int(block_table[b][j // P])
                kv_pages[to, :, h, i % P] = old_pages[frm, :, h, j % P]
                kv_weights[to, h, i % P] = old_weights[frm, h, j % P]
