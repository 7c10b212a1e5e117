"""GPU tests of chunked prefill over a cache of 4-bit codes against the oracle (oracle/fp4.py), chunk by chunk with the quantising append: outputs to bounds that
follow from what is rounded, the cache bit for bit.  Slots that hold no token have exponents that stand for NaN: a stray read of one would show."""
import numpy as np
import pytest
import torch

from oracle import fp4
from oracle import packer as opacker
from paper_2401_11181_amd import synth, tetri
from paper_2401_11181_amd.prefill import ChunkedPrefill
import gpu_common as gc
from fp4_common import DEV, bf16, cache, check, dev, f64
from test_gpu_parity import CASES, VARIANTS

pytestmark = pytest.mark.gpu


@pytest.fixture(params=VARIANTS + [3], ids=["auto", "wave4", "wave8", "tails", "tails-wave4", "whole", "tails-half", "stream5", "stream5-wave4", "stream2", "stream200", "small-tiles"])
def variant(request):
    return request.param


def empty_pool(w):
    pool = np.zeros((w.num_pages, 2, w.num_kv_heads, fp4.slab_bytes(w.head_dim)), dtype=np.uint8)
    pool[..., fp4.P * w.head_dim // 2:] = 255
    return pool


_oracle_runs = {}


def oracle_run(w, qs, ks, vs, tables):
    """Outputs and spreads per request, and the cache, computed once for all kernel variants."""
    key = (w.name, w.seed, w.scale)
    if key not in _oracle_runs:
        pool = empty_pool(w)
        outs, spreads = [np.zeros(tuple(t.shape)) for t in qs], [np.zeros(tuple(t.shape)) for t in qs]
        blocks = max(len(t) for t in tables)
        for segs in opacker.pack_chunks(w.prompt_lens, w.order, w.chunk_size):
            cu, ctx = opacker.chunk_arrays(segs)
            bt = np.zeros((len(segs), blocks), dtype=np.int32)
            for i, (req, _s, _n) in enumerate(segs):
                bt[i, :len(tables[req])] = tables[req]
            rows = lambda per: np.concatenate([f64(per[req][start:start + n]) for req, start, n in segs])
            q, k, v = rows(qs), rows(ks), rows(vs)
            o, d = fp4.attention(q, k, v, pool, bt, cu, ctx, w.scale)
            fp4.append(k, v, pool, bt, cu, ctx)
            for i, (req, start, n) in enumerate(segs):
                outs[req][start:start + n], spreads[req][start:start + n] = o[cu[i]:cu[i] + n], d[cu[i]:cu[i] + n]
        _oracle_runs[key] = outs, spreads, pool
    return _oracle_runs[key]


def gpu_run(w, qs, ks, vs, tables, variant=0, pad_fill=None):
    sess = ChunkedPrefill(w.prompt_lens, w.order, w.chunk_size, w.num_q_heads, w.num_kv_heads, w.head_dim, w.num_pages, tables, device=DEV)
    gc.set_variant(sess, variant)
    pool = dev(empty_pool(w))
    dq, dk, dv = [[t.to(DEV) for t in x] for x in (qs, ks, vs)]
    outs = [torch.zeros_like(t) for t in qs]
    for c in range(sess.n_chunks):
        q, k, v = [sess.gather_chunk(x, c) for x in (dq, dk, dv)]
        segs = sess.chunk_segments(c)
        real = sum(n for _, _, n in segs)
        if pad_fill is not None:
            q[real:], k[real:], v[real:] = pad_fill, pad_fill, pad_fill
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
        sess.attn_fp4(c, q, k, v, pool, w.scale, 1, out)
        torch.cuda.synchronize()
        o, at = out.cpu(), 0
        for req, start, n in segs:
            outs[req][start:start + n] = o[at:at + n]
            at += n
        assert (o[real:].view(torch.int16) == 0).all(), "padding rows of out must be +0"
    return outs, pool, sess


def run_case(w, variant, scores=1.0):
    qs, ks, vs, tables = gc.workload_tensors(w)
    outs, pool, _ = gpu_run(w, qs, ks, vs, tables, variant)
    ref, spread, want = oracle_run(w, qs, ks, vs, tables)
    for r in range(len(outs)):
        check(outs[r], ref[r], spread[r], "%s request %d" % (w.name, r), scores)
    assert np.array_equal(pool.cpu().numpy(), want), w.name + ": the cache differs from the oracle's"


@pytest.mark.parametrize("name", sorted(CASES))
def test_shapes(name, variant):
    lens, chunk, hq, hkv, d = CASES[name]
    run_case(synth.small("fp4-" + name, lens, chunk, hq, hkv, d, seed=500 + sorted(CASES).index(name)), variant)


def test_more_than_64_segments_in_a_chunk(variant):
    rng = np.random.default_rng(152)
    run_case(synth.small("fp4-many-segments", [int(x) for x in rng.integers(1, 5, size=150)], 256, 4, 2, 128, seed=552), variant)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.7])
def test_softmax_scales(scale, variant):
    run_case(synth.small("fp4-scale", [200, 45], 64, 2, 2, 64, seed=532, scale=scale), variant, scores=max(1.0, 8 * abs(scale)))


def test_without_append_the_pool_is_only_read(variant):
    w = synth.small("fp4-read-only", [300, 90], 128, 4, 2, 128, seed=533)
    qs, ks, vs, tables = gc.workload_tensors(w)
    _, pool, sess = gpu_run(w, qs, ks, vs, tables, variant)
    c = sess.n_chunks - 1
    q, k, v = [sess.gather_chunk([t.to(DEV) for t in x], c) for x in (qs, ks, vs)]
    before, a, b = pool.clone(), torch.zeros_like(q), torch.zeros_like(q)
    sess.attn_fp4(c, q, k, v, pool, w.scale, 0, a)
    torch.cuda.synchronize()
    assert torch.equal(pool, before)
    sess.attn_fp4(c, q, k, v, pool, w.scale, 1, b)                  # rewrites the bytes the chain wrote
    torch.cuda.synchronize()
    assert torch.equal(pool, before) and torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("fill", [3.0e4, float("nan")])
def test_padding_rows_are_inert(fill, variant):
    w = synth.small("fp4-pad", [100, 37], 64, 2, 2, 128, seed=534)
    qs, ks, vs, tables = gc.workload_tensors(w)
    ref, pool_ref, _ = gpu_run(w, qs, ks, vs, tables, variant)
    out, pool, _ = gpu_run(w, qs, ks, vs, tables, variant, pad_fill=fill)
    assert all(torch.equal(x, y) for x, y in zip(ref, out)) and torch.equal(pool_ref, pool)


def test_powers_of_both_sides(variant):
    """Groups of K and V under powers of their own from 2^-6 up, entries of the block table behind a segment's pages that must not be used."""
    rng = np.random.default_rng(535)
    hq, hkv, d = 8, 2, 128
    ctx, n = [100, 0, 333], [40, 17, 60]
    pool, bt = cache(rng, ctx, hkv, d, extra=60)
    at = fp4.P * d // 2
    live = pool[..., at:] != 255
    pool[..., at:][live] = (127 + rng.integers(-6, 2, size=live.sum())).astype(np.uint8)
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    q, k, v = bf16(rng, 128, hq, d), bf16(rng, 128, hkv, d), bf16(rng, 128, hkv, d)
    h = tetri.Tetri(hq, hkv, d, 128, len(pool), bt.shape[1], 8)
    gc.set_variant(type("Session", (), {"handle": h}), variant)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    h.tetri_chunk_prefill_attn_fp4(dev(q), dev(k), dev(v), dev(pool), dev(bt), dev(cu), dev(np.array(ctx, dtype=np.int32)), 3, 0.05, 0, out)
    torch.cuda.synchronize()
    ref, spread = fp4.attention(f64(q), f64(k), f64(v), pool, bt, cu, ctx, 0.05)
    check(out, ref, spread, scores=4.0)


def test_replayed():
    """A captured chunk with append, replayed over contexts that grow; its rows' codes and outputs are the eager ones each time."""
    w = synth.small("fp4-replay", [256], 64, 4, 2, 128, seed=536)
    qs, ks, vs, tables = gc.workload_tensors(w)
    eager, pool_ref, sess = gpu_run(w, qs, ks, vs, tables)
    pool = dev(empty_pool(w))
    q, k, v = [sess.gather_chunk([t.to(DEV) for t in x], 0) for x in (qs, ks, vs)]
    ctx, out = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros_like(q)
    cu, _ctx, bt, _S = sess.meta[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sess.handle.tetri_chunk_prefill_attn_fp4(q, k, v, pool, bt, cu, ctx, 1, w.scale, 1, out)
    pool.copy_(dev(empty_pool(w)))
    for c in range(sess.n_chunks):
        for to, x in zip((q, k, v), (qs, ks, vs)):
            to.copy_(sess.gather_chunk([t.to(DEV) for t in x], c))
        ctx.fill_(64 * c)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu().view(torch.int16), eager[0][64 * c:64 * c + 64].view(torch.int16))
    assert torch.equal(pool, pool_ref)


def test_refusals():
    h = tetri.Tetri(4, 2, 128, 64, 8, 4, 4)
    q, k = torch.zeros((64, 4, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((64, 2, 128), dtype=torch.bfloat16, device=DEV)
    pool = torch.zeros((8, 2, 2, fp4.slab_bytes(128)), dtype=torch.uint8, device=DEV)
    bt, cu, ctx = [torch.zeros(8, dtype=torch.int32, device=DEV) for _ in range(3)]
    good = dict(q=q, k_new=k, v_new=k, kv_pages_fp4=pool, block_table=bt, cu_chunk_q_lens=cu, ctx_lens=ctx, num_segs=1, scale=0.1, append=0, out=q.clone())
    for x in (dict(append=2), dict(append=-1), dict(kv_pages_fp4=None), dict(kv_pages_fp4=pool.view(-1)[1:]), dict(num_segs=0), dict(num_segs=5),
              dict(scale=float("nan")), dict(cu_chunk_q_lens=None), dict(block_table=None), dict(q=None), dict(out=q.view(-1)[1:])):
        with pytest.raises(tetri.TetriError) as e:
            h.tetri_chunk_prefill_attn_fp4(**{**good, **x})
        assert e.value.status == tetri.TETRI_ERR_INVALID_ARG, x
