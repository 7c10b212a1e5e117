"""Ways of calling: a scheduled batch over codes and with replaced metadata, two streams at once, graphs."""
import numpy as np
import pytest
import torch

from oracle import evict
from paper_2401_11181_amd.prefill import ChunkedPrefill
import evict_common as ec
import gpu_common as gc
from test_gpu_evict import dev, fill_weights, handle, workspace

pytestmark = pytest.mark.gpu
DEV = gc.DEV


@pytest.mark.parametrize("replaced", [False, True], ids=["planned", "replaced"])
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_weights_of_a_scheduled_batch(fp8, replaced):
    """`replaced`: entries of `meta` that the plan does not know, so that the longest context is not known either."""
    hq, hkv, d, C, scale = 4, 2, 64, 48, 0.125
    prompts = [70, 33, 90]
    c = ec.Cache([0, 0, 0], hkv, d, 500, fp8, room=prompts, extra_blocks=0)
    sess = ChunkedPrefill(prompts, None, C, hq, hkv, d, c.pages, [list(c.bt[b, :-(-n // 16)]) for b, n in enumerate(prompts)])
    if replaced:
        sess.meta = [tuple(t.clone() for t in m[:3]) + (m[3],) for m in sess.meta]
    gen = torch.Generator().manual_seed(501)
    q, k, v = ([torch.randn((m, n, d), generator=gen).to(torch.bfloat16) for m in prompts] for n in (hq, hkv, hkv))
    pool, w = dev(c.pool), dev(c.weights.clone())
    want, amp = c.weights.double().numpy(), 0.0
    for chunk in range(sess.n_chunks):
        cq, ck, cv = (sess.gather_chunk([dev(t) for t in x], chunk) for x in (q, k, v))
        segs = sess.chunk_segments(chunk)
        cu = np.concatenate([[0], np.cumsum([n for _, _, n in segs])])
        c.pool = pool.cpu()
        evict.prefill_weights(cq.cpu().double().numpy(), ck.cpu().double().numpy(), c.float_pool(), want, c.bt[[r for r, _, _ in segs]], cu,
                              [start for _, start, _ in segs], 16, scale)
        work = workspace(sess.weights_workspace(chunk, 16))
        sess.weights(chunk, cq, ck, pool, w, scale, 16, work, ec.K_SCALE if fp8 else None)
        if fp8:
            sess.attn_fp8(chunk, cq, ck, cv, pool, scale, ec.K_SCALE, ec.V_SCALE, 1, torch.zeros_like(cq))
        else:
            sess.append(chunk, ck, cv, pool)
    for x in q:
        amp = max(amp, ec.amplitude(x.double().numpy().reshape(-1, d), np.concatenate([t.double().numpy().reshape(-1, d) for t in k]), scale))
    got = w.cpu().double().numpy()
    for b, n in enumerate(prompts):
        pages, places = c.slots(b, n)
        g, ref = got[pages, :, places], want[pages, :, places]
        # (a code is off by at most 1/16 of its value, and so is the sum of absolute products; three chunks add to a slot)
        bound = ec.weight_bound(ref, 0.0, amp * (1.0625 if fp8 else 1.0), d) + 3 * ref * 2.0 ** -24
        assert (np.abs(g - ref) <= bound).all()


def test_two_streams_at_once():
    """Weighing, choice and moves of two sets of requests, each on a stream of its own with a workspace of its own."""
    hq, hkv, d, keep, recent, last = 8, 2, 128, 500, 40, 30
    h, sides = None, []
    for seed in (510, 520):
        c = ec.Cache([1300, 900], hkv, d, seed, room=30)
        h = h or handle(c, hq)
        gen = torch.Generator().manual_seed(seed + 1)
        q, k = (torch.randn((64, n, d), generator=gen).to(torch.bfloat16).to(DEV) for n in (hq, hkv))
        sides.append((c, q, k, dev(c.bt), dev(c.ctx), dev(np.array([0, 30, 60], dtype=np.int32)),
                      workspace(h.tetri_chunk_prefill_weights_workspace(2, 1300, last))))

    def calls(side, stream=None):
        c, q, k, bt, ctx, cu, work = side
        pool, w = dev(c.pool.clone()), dev(torch.nan_to_num(c.weights))
        slots, lens = torch.zeros((2, hkv, keep), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
        torch.cuda.synchronize()

        def run():
            h.tetri_chunk_prefill_weights(q, k, pool, w, bt, cu, ctx, 2, 1300, last, 0.09, 0, 1.0, work, work.numel(), stream)
            h.tetri_kv_select(w, bt, ctx, 2, 1300, keep, recent, slots, lens, stream)
            h.tetri_kv_compact(slots, bt, ctx, 2, keep, recent, pool, w, 0, stream)
        return run, (pool, w, slots, lens)

    want = []
    for side in sides:
        run, got = calls(side)
        run()
        torch.cuda.synchronize()
        want.append(got)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        both = [calls(side, stream) for side, stream in zip(sides, streams)]
        for run, _ in both:
            run()
        torch.cuda.synchronize()
        for (_, got), ref in zip(both, want):
            for a, b in zip(got, ref):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    h.close()


@pytest.mark.parametrize("bound", [3000, 40000, 1 << 19])
def test_choice_captured_under_any_bound(bound):
    """The kernel for many slots asks for more LDS than others: that, too, in a graph."""
    c = ec.Cache([2500, 70], 2, 64, 530, extra_blocks=(1 << 19) // 16)
    fill_weights(c, "spread", 531)
    h = handle(c, 2)
    w, bt, ctx = dev(c.weights), dev(c.bt), dev(c.ctx)
    slots, lens = torch.zeros((2, 2, 300), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.tetri_kv_select(w, bt, ctx, 2, bound, 300, 20, slots, lens)
    for turn in range(3):
        fill_weights(c, "spread", 532 + turn)
        w.copy_(dev(c.weights))
        slots.zero_(), lens.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want, want_lens = evict.select(c.weights.numpy(), c.bt, c.lens, 300, 20)
        assert np.array_equal(slots.cpu().numpy(), want) and lens.tolist() == want_lens.tolist()
        h.tetri_kv_select(w, bt, ctx, 2, bound, 100, 20, slots, lens)        # eager, in between
    h.close()
