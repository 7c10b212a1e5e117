"""Weights of tokens that come into the cache by calls that do not weigh: what include/tetri.h asks the caller to write is enough."""
import numpy as np
import pytest
import torch

from oracle import evict
import evict_common as ec
import gpu_common as gc
from test_gpu_evict import dev, handle, workspace

pytestmark = pytest.mark.gpu
DEV = gc.DEV
HQ, HKV, D, SCALE = 4, 2, 64, 0.125


class Run:
    """Requests of which nothing is cached yet, in a pool and weights of garbage; calls of the library beside the oracle's."""

    def __init__(self, tokens, seed, fp8):
        self.c = c = ec.Cache([0] * len(tokens), HKV, D, seed, fp8, room=tokens, extra_blocks=0)
        self.gen, self.fp8, self.B = torch.Generator().manual_seed(seed + 1), int(fp8), len(tokens)
        self.pool, self.w, self.bt = dev(c.pool.clone()), dev(c.weights.clone()), dev(c.bt)
        self.want = c.weights.double().numpy()                # (NaN where nothing has been written)
        self.lens = [0] * self.B
        self.h = handle(c, HQ, 64, 8)
        most = c.blocks * ec.PAGE - 1
        self.work = workspace(max(self.h.tetri_decode_attn_weights_workspace(self.B, most), self.h.tetri_chunk_prefill_weights_workspace(self.B, most, 64)))

    def zero(self, b, first, last):
        """Slots [first, last) of request b, both here and in the oracle's weights."""
        pages, places = (x[first:last] for x in self.c.slots(b, last))
        self.w[dev(pages.astype(np.int64)), :, dev(places)] = 0.0
        self.want[pages, :, places] = 0.0

    def zero_pages(self):
        for b in range(self.B):
            pages = np.unique(self.c.bt[b][self.c.bt[b] < self.c.pages])
            self.w[dev(pages.astype(np.int64))] = 0.0
            self.want[pages] = 0.0

    def values(self, n, heads):
        return torch.randn((n, heads, D), generator=self.gen).to(torch.bfloat16)

    def float_pool(self):
        self.c.pool = self.pool.cpu()
        return self.c.float_pool()

    def prefill(self, rows, weighed):
        cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        q, k, v = self.values(64, HQ), self.values(64, HKV), self.values(64, HKV)
        ctx = np.array(self.lens, dtype=np.int32)
        args = (dev(q), dev(k), dev(v), self.pool, self.bt, dev(cu), dev(ctx), self.B, SCALE)
        if weighed:
            evict.prefill_weights(q.double().numpy(), k.double().numpy(), self.float_pool(), self.want, self.c.bt, cu, self.lens, 64, SCALE)
            self.h.tetri_chunk_prefill_weights(args[0], args[1], self.pool, self.w, self.bt, args[5], args[6], self.B, max(self.lens), 64, SCALE, self.fp8,
                                               ec.K_SCALE, self.work, self.work.numel())
        out = torch.zeros((64, HQ, D), dtype=torch.bfloat16, device=DEV)
        if self.fp8:
            self.h.tetri_chunk_prefill_attn_fp8(*args, ec.K_SCALE, ec.V_SCALE, 1, out)
        else:
            self.h.tetri_chunk_prefill_attn_append(*args, out)
        self.lens = [n + m for n, m in zip(self.lens, rows)]

    def decode(self, weighed, append=1):
        q, k, v = self.values(self.B, HQ), self.values(self.B, HKV), self.values(self.B, HKV)
        out, ctx = torch.zeros((self.B, HQ, D), dtype=torch.bfloat16, device=DEV), dev(np.array(self.lens, dtype=np.int32))
        args = (dev(q), dev(k), dev(v), self.pool)
        if weighed:
            evict.decode_weights(q.double().numpy(), k.double().numpy(), self.float_pool(), self.want, self.c.bt, self.lens, SCALE, append)
            self.h.tetri_decode_attn_weights(*args, self.w, self.bt, ctx, self.B, max(self.lens), SCALE, append, self.fp8, ec.K_SCALE, ec.V_SCALE,
                                             self.work, self.work.numel(), out)
        elif self.fp8:
            self.h.tetri_decode_attn_fp8(*args, self.bt, ctx, self.B, max(self.lens), SCALE, ec.K_SCALE, ec.V_SCALE, append, out)
        else:
            self.h.tetri_decode_attn_append(*args, self.bt, ctx, self.B, max(self.lens), SCALE, out)
        if not append:                                       # by a call of its own
            self.h.tetri_kv_append(args[1], args[2], self.pool, self.bt, dev(np.arange(self.B + 1, dtype=np.int32)), ctx, self.B)
        self.lens = [n + 1 for n in self.lens]

    def cut(self, keep, recent):
        """The choice by the weights as the library has them; the oracle follows it."""
        slots, lens = torch.zeros((self.B, HKV, keep), dtype=torch.int32, device=DEV), torch.zeros(self.B, dtype=torch.int32, device=DEV)
        ctx = dev(np.array(self.lens, dtype=np.int32))
        self.h.tetri_kv_select(self.w, self.bt, ctx, self.B, max(self.lens), keep, recent, slots, lens)
        scratch = np.zeros(self.c.pool.shape, dtype=np.uint8)
        evict.compact(slots.cpu().numpy(), self.c.bt, self.lens, keep, scratch, self.want)
        self.h.tetri_kv_compact(slots, self.bt, ctx, self.B, keep, recent, self.pool, self.w, self.fp8)
        old, self.lens = self.lens, lens.tolist()
        return old

    def check(self):
        got = self.w.cpu().double().numpy()
        for b in range(self.B):
            pages, places = self.c.slots(b, self.lens[b])
            g, w = got[pages, :, places], self.want[pages, :, places]
            assert np.isfinite(g).all()
            # (some hundred terms, all positive; 64 products a score: see evict_common)
            assert np.allclose(g, w, rtol=1e-4, atol=1e-7), np.abs(g - w).max()


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_pages_of_zeros_and_calls_that_do_not_weigh(fp8):
    r = Run([90, 60], 400, fp8)
    r.zero_pages()
    r.prefill([30, 33], False)
    r.prefill([25, 10], True)
    r.decode(False)
    r.decode(True)
    if not fp8:
        r.decode(True, append=0)
    r.decode(True)
    r.check()
    r.h.close()


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_tokens_cached_behind_a_cut(fp8):
    """The slots that were given up hold old weights: they are written to before a token is cached there by a call that does not weigh."""
    r = Run([90, 60], 410, fp8)
    r.prefill([34, 30], True)                                # (weighed from the first token on: no slot needs a value)
    r.prefill([40, 20], True)
    r.decode(True)
    old = r.cut(32, 8)
    assert old == [75, 51] and r.lens == [32, 32]
    for b in range(2):
        r.zero(b, 32, old[b])
    r.decode(False)
    r.prefill([20, 7], False)
    r.decode(True)
    r.check()
    r.h.close()


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_tokens_weighed_behind_a_cut(fp8):
    """A token that comes by a weighing call gets its weight from that call, whatever its slot held."""
    r = Run([90, 60], 415, fp8)
    r.prefill([34, 30], True)
    r.prefill([25, 20], True)
    r.cut(32, 8)
    r.w[:, :, :] = torch.where(torch.isnan(r.w), 1e9, r.w)
    for _ in range(3):
        r.decode(True)
    r.prefill([20, 15], True)
    r.check()
    r.h.close()


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_weights_follow_a_request_to_another_pool(fp8):
    """Weighed while it is prefilled, exported, imported at other pages with its weights, decoded there."""
    src, dst = Run([70, 41], 420, fp8), Run([90, 60], 430, fp8)
    src.prefill([34, 30], True)
    src.prefill([30, 11], True)
    cu, total = dev(np.array([0, 64, 105], dtype=np.int32)), 105
    buf = torch.zeros(2 * HKV * D * total * 2, dtype=torch.uint8, device=DEV)
    if fp8:
        # (a pool of codes is carried page by page like the weights: the quantising export starts from a 16-bit pool)
        for b, n in enumerate(src.lens):
            blocks = -(-n // ec.PAGE)
            dst.pool[dst.bt[b, :blocks].long()] = src.pool[src.bt[b, :blocks].long()]
    else:
        src.h.tetri_kv_export(src.pool, src.bt, cu, None, 2, total, buf)
        dst.h.tetri_kv_import(buf, dst.bt, cu, None, 2, total, dst.pool)
    for b, n in enumerate(src.lens):
        blocks = -(-n // ec.PAGE)
        dst.w[dst.bt[b, :blocks].long()] = src.w[src.bt[b, :blocks].long()]
        dst.want[dst.c.bt[b, :blocks]] = src.want[src.c.bt[b, :blocks]]
    dst.lens = list(src.lens)
    for _ in range(3):
        dst.decode(True)
    dst.check()
    src.h.close(), dst.h.close()


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_requests_that_share_a_prefix(fp8):
    """Weighed by calls one after the other: what both give to the prefix adds up."""
    r = Run([80, 80], 440, fp8)
    r.c.bt[1, :2] = r.c.bt[0, :2]                            # 32 tokens
    r.bt = dev(r.c.bt)
    ones = [r.c.bt[b:b + 1].copy() for b in range(2)]

    def alone(b, call):
        r.c.bt, r.B, whole = ones[b], 1, (r.bt, r.lens)
        r.bt, r.lens = dev(ones[b]), [r.lens[b]]
        call()
        whole[1][b] = r.lens[0]
        r.bt, r.lens = whole
        r.c.bt, r.B = np.concatenate(ones), 2

    alone(0, lambda: r.prefill([32], True))
    r.lens[1] = 32
    for b, n in ((0, 10), (1, 21)):
        alone(b, lambda: r.prefill([n], True))
    for _ in range(3):
        for b in range(2):
            alone(b, lambda: r.decode(True))
    assert r.lens == [45, 56]
    r.check()
    r.h.close()
