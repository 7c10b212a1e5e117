"""GPU tests of the operators over 4-bit codes and of the norm and rotation as a server runs them: one after the other on the same cache, from two graphs that share a
handle, on other streams, over large batches and pools.  Every link is checked against its definition on the inputs that it was given."""
import numpy as np
import pytest
import torch

from oracle import fp4
from oracle import rope as orope
from paper_2401_11181_amd import tetri
from paper_2401_11181_amd.prefill import ChunkedPrefill
from fp4_common import DEV, STEP, bf16, cache, check, dev, f64
from test_gpu_rope import check as check_rope, sizes

pytestmark = pytest.mark.gpu
P = fp4.P


class Server:
    """A few requests of a model's one layer: projections' rows, weights of the norm, pages."""

    def __init__(self, hq, hkv, d, prompts, new, chunk, seed):
        self.hq, self.hkv, self.d, self.prompts, self.scale = hq, hkv, d, prompts, d ** -0.5
        self.rng = rng = np.random.default_rng(seed)
        need = [-(-(n + new) // P) for n in prompts]
        self.pages, perm, at = sum(need) + 2, rng.permutation(sum(need) + 2), 0
        self.tables = []
        for n in need:
            self.tables.append([int(x) for x in perm[at:at + n]])
            at += n
        self.bt = np.full((len(prompts), max(need)), perm[-1], dtype=np.int32)
        for r, t in enumerate(self.tables):
            self.bt[r, :len(t)] = t
        self.w = [bf16(rng, d) * 0.2 + 1.0 for _ in range(2)]
        self.freq = (10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
        self.rope = tetri.Rope(self.freq)
        self.sess = ChunkedPrefill(prompts, list(range(len(prompts))), chunk, hq, hkv, d, self.pages, self.tables, device=DEV)
        self.rows = [dev(bf16(rng, n, (hq + 2 * hkv) * d)) for n in prompts]

    def parts(self, x):
        a, b = self.hq * self.d, (self.hq + self.hkv) * self.d
        return x[:, :a], x[:, a:b], x[:, b:].reshape(len(x), self.hkv, self.d).contiguous()

    def check_rotation(self, x, got, heads, weight, positions):
        x = f64(x.cpu()).reshape(len(positions), heads, self.d)
        ref = orope.qk_norm_rope(x, f64(weight), 1e-6, self.freq, np.zeros(len(self.freq), dtype=int), np.array(positions)[None], False)
        check_rope(got, ref, sizes(x, f64(weight), 1e-6, len(self.freq), False))

    def chunk(self, c):
        """Rotated q and k and the v of chunk c, checked; its segments."""
        q, k, v = self.parts(self.sess.gather_chunk(self.rows, c))
        q_out = torch.zeros((len(q), self.hq, self.d), dtype=torch.bfloat16, device=DEV)
        k_out = torch.zeros((len(q), self.hkv, self.d), dtype=torch.bfloat16, device=DEV)
        self.sess.qk_norm_rope(c, q, k, dev(self.w[0]), dev(self.w[1]), 1e-6, self.rope, q_out, k_out)
        torch.cuda.synchronize()
        segs = self.sess.chunk_segments(c)
        positions = np.concatenate([start + np.arange(n) for _, start, n in segs])
        real = len(positions)
        for x, got, heads, w in ((q, q_out, self.hq, self.w[0]), (k, k_out, self.hkv, self.w[1])):
            self.check_rotation(x[:real], got[:real], heads, w, positions)
            assert not got[real:].any()
        return q_out, k_out, v, segs

    def token(self, handle, lens):
        """The same of one new token of every request behind `lens` tokens."""
        B = len(lens)
        q, k, v = self.parts(dev(bf16(self.rng, B, (self.hq + 2 * self.hkv) * self.d)))
        q_out = torch.zeros((B, self.hq, self.d), dtype=torch.bfloat16, device=DEV)
        k_out = torch.zeros((B, self.hkv, self.d), dtype=torch.bfloat16, device=DEV)
        pos = dev(np.array(lens, dtype=np.int32)[None])
        handle.tetri_qk_norm_rope(q, q.stride(0), k, k.stride(0), dev(self.w[0]), dev(self.w[1]), 1e-6, self.rope, pos, None, None, 0, B, q_out, k_out)
        torch.cuda.synchronize()
        self.check_rotation(q, q_out, self.hq, self.w[0], lens)
        self.check_rotation(k, k_out, self.hkv, self.w[1], lens)
        return q_out, k_out, v

    def decode(self, handle, pool, bt, known, lens, steps):
        """Some tokens more, cached in codes.  known: the pool as the oracle has it, kept up with."""
        d_bt = dev(bt)
        for _ in range(steps):
            q, k, v = self.token(handle, lens)
            out = torch.zeros_like(q)
            handle.tetri_decode_attn_fp4(q, k, v, pool, d_bt, dev(np.array(lens, dtype=np.int32)), len(lens), max(lens), self.scale, 1, out)
            torch.cuda.synchronize()
            q, k, v = [f64(x.cpu()) for x in (q, k, v)]
            cu = np.arange(len(lens) + 1)
            check(out, *fp4.attention(q, k, v, known, bt, cu, lens, self.scale), "decode", scores=4.0)
            fp4.append(k, v, known, bt, cu, lens)
            assert np.array_equal(pool.cpu().numpy(), known)
            lens = [n + 1 for n in lens]


def empty(pages, hkv, d):
    pool = np.zeros((pages, 2, hkv, fp4.slab_bytes(d)), dtype=np.uint8)
    pool[..., P * d // 2:] = 255
    return pool


SERVERS = {"mha": (3, 3, 128), "gqa": (8, 2, 128), "gqa-d64": (6, 2, 64)}


@pytest.mark.parametrize("name", sorted(SERVERS))
def test_prompts_in_16_bits_then_codes(name):
    """Prefill over the 16-bit cache, export of the prompts in codes, import on another instance with other pages, which generates."""
    s = Server(*SERVERS[name], [70, 5, 150, 1], 4, 64, 301)
    pool = torch.zeros((s.pages, 2, s.hkv, P, s.d), dtype=torch.bfloat16, device=DEV)
    want = np.zeros(tuple(pool.shape))
    for c in range(s.sess.n_chunks):
        q, k, v, segs = s.chunk(c)
        out = torch.zeros_like(q)
        s.sess.attn_append(c, q, k, v, pool, s.scale, out)
        torch.cuda.synchronize()
        k, v, at = f64(k.cpu()), f64(v.cpu()), 0
        for req, start, n in segs:
            for t in range(n):
                page = s.tables[req][(start + t) // P]
                want[page, 0, :, (start + t) % P], want[page, 1, :, (start + t) % P] = k[at + t], v[at + t]
            at += n
    assert np.array_equal(f64(pool.cpu()), want)
    cu = np.concatenate([[0], np.cumsum(s.prompts)]).astype(np.int32)
    buf = torch.full((2 * s.hkv * int(cu[-1]) * (s.d // 2 + s.d // 32),), 99, dtype=torch.uint8, device=DEV)
    s.sess.handle.tetri_kv_export_fp4(pool, dev(s.bt), dev(cu), None, len(s.prompts), int(cu[-1]), buf)
    bt = np.full_like(s.bt, s.pages)
    perm, at = s.rng.permutation(s.pages), 0
    for r, t in enumerate(s.tables):
        bt[r, :len(t)] = perm[at:at + len(t)]
        at += len(t)
    other = tetri.Tetri(s.hq, s.hkv, s.d, 64, s.pages + 1, bt.shape[1], 8)
    known = empty(s.pages + 1, s.hkv, s.d)
    codes = dev(known)
    other.tetri_kv_import_fp4(buf, dev(bt), dev(cu), None, len(s.prompts), int(cu[-1]), codes)
    torch.cuda.synchronize()
    data = fp4.export(want, s.bt, cu)
    assert np.array_equal(buf.cpu().numpy(), data)
    fp4.import_(data, known, bt, cu, None, s.d)
    assert np.array_equal(codes.cpu().numpy(), known)
    s.decode(other, codes, bt, known, list(s.prompts), 3)


@pytest.mark.parametrize("name", sorted(SERVERS))
def test_codes_from_the_first_chunk_on(name):
    """Prefill over the cache of codes with append, then decode on it."""
    s = Server(*SERVERS[name], [130, 3, 90], 3, 64, 302)
    known = empty(s.pages, s.hkv, s.d)
    pool = dev(known)
    for c in range(s.sess.n_chunks):
        q, k, v, segs = s.chunk(c)
        out = torch.zeros_like(q)
        s.sess.attn_fp4(c, q, k, v, pool, s.scale, 1, out)
        torch.cuda.synchronize()
        q, k, v = [f64(x.cpu()) for x in (q, k, v)]
        cu = np.concatenate([[0], np.cumsum([n for _, _, n in segs])])
        ctx, bt = [start for _, start, _ in segs], np.stack([s.bt[req] for req, _, _ in segs])
        check(out, *fp4.attention(q, k, v, known, bt, cu, ctx, s.scale), "chunk %d" % c, scores=4.0)
        fp4.append(k, v, known, bt, cu, ctx)
        assert np.array_equal(pool.cpu().numpy(), known)
    s.decode(s.sess.handle, pool, s.bt, known, list(s.prompts), 3)


def test_two_graphs_of_one_handle():
    """A decode iteration cut in ranges and a chunk on the small tiles, captured on one handle, whose scratch memory they share: replayed in turn with eager calls of both between
    them, every result that of the first time."""
    rng = np.random.default_rng(303)
    hq, hkv, d = 8, 2, 128
    lens, ctx = [700, 3, 260, 90], [400, 0, 33]
    pool, bt = cache(rng, lens + ctx, hkv, d, extra=60)
    h = tetri.Tetri(hq, hkv, d, 128, len(pool), bt.shape[1], 8)
    h.tetri_set_option("decode_ranges", 9)
    h.tetri_set_option("attn_variant", 3)
    d_pool = dev(pool)
    q, k, v = dev(bf16(rng, 4, hq, d)), dev(bf16(rng, 4, hkv, d)), dev(bf16(rng, 4, hkv, d))
    cq, ck, cv = dev(bf16(rng, 128, hq, d)), dev(bf16(rng, 128, hkv, d)), dev(bf16(rng, 128, hkv, d))
    a, b = torch.zeros_like(q), torch.zeros_like(cq)
    bt_a, bt_b = dev(bt[:4]), dev(bt[4:])
    lens_a, ctx_b, cu = dev(np.array(lens, dtype=np.int32)), dev(np.array(ctx, dtype=np.int32)), dev(np.array([0, 40, 57, 110], dtype=np.int32))

    def decode():
        h.tetri_decode_attn_fp4(q, k, v, d_pool, bt_a, lens_a, 4, 700, 0.09, 0, a)

    def chunk():
        h.tetri_chunk_prefill_attn_fp4(cq, ck, cv, d_pool, bt_b, cu, ctx_b, 3, 0.09, 0, b)
    decode(), chunk()
    torch.cuda.synchronize()
    check(a, *fp4.attention(f64(q.cpu()), f64(k.cpu()), f64(v.cpu()), pool, bt[:4], np.arange(5), lens, 0.09))
    check(b, *fp4.attention(f64(cq.cpu()), f64(ck.cpu()), f64(cv.cpu()), pool, bt[4:], [0, 40, 57, 110], ctx, 0.09))
    first = a.clone(), b.clone()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, f in zip(graphs, (decode, chunk)):
        with torch.cuda.graph(g):
            f()
    for turn in (0, 1, 0, 0, 1, "decode", 1, "chunk", 0, 1, "chunk", "decode", 0, 1, 1):
        a.zero_(), b.fill_(3.0)
        if turn == "decode":
            decode()
        elif turn == "chunk":
            chunk()
        else:
            graphs[turn].replay()
        torch.cuda.synchronize()
        if turn in (0, "decode"):
            assert torch.equal(a.view(torch.int16), first[0].view(torch.int16)) and (b == 3.0).all(), turn
        else:
            assert torch.equal(b.view(torch.int16), first[1].view(torch.int16)) and not a.any(), turn


def test_on_another_stream():
    """Every call on a stream of its own, behind work that makes its inputs there."""
    rng = np.random.default_rng(304)
    hq, hkv, d, lens = 4, 2, 128, [100, 40]
    pool, bt = cache(rng, lens, hkv, d, extra=20)
    h = tetri.Tetri(hq, hkv, d, 64, len(pool), bt.shape[1], 8)
    rows, q, k, v = [bf16(rng, len(pool), 2, hkv, P, d), bf16(rng, 64, hq, d), bf16(rng, 64, hkv, d), bf16(rng, 64, hkv, d)]
    cu, first = np.array([0, 11, 31], dtype=np.int32), dev(np.array([3, 0], dtype=np.int32))
    src = [dev(x) for x in (pool, rows, q, k, v)]
    d_bt, d_cu, d_lens = dev(bt), dev(cu), dev(np.array(lens, dtype=np.int32))
    dst = [torch.zeros_like(x) for x in src]
    buf = torch.zeros(2 * hkv * 31 * (d // 2 + d // 32), dtype=torch.uint8, device=DEV)
    a, b = torch.zeros_like(src[2][:2]), torch.zeros_like(src[2])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for to, x in zip(dst, src):
            to.copy_(x)
    codes, pages, q1, k1, v1 = dst
    h.tetri_chunk_prefill_attn_fp4(q1, k1, v1, codes, d_bt, d_cu, d_lens, 2, 0.1, 0, b, side)
    h.tetri_decode_attn_fp4(q1, k1, v1, codes, d_bt, d_lens, 2, 100, 0.1, 0, a, side)
    h.tetri_kv_export_fp4(pages, d_bt, d_cu, first, 2, 31, buf, side)
    h.tetri_kv_import_fp4(buf, d_bt, d_cu, first, 2, 31, codes, side)
    side.synchronize()
    x = [f64(y) for y in (q, k, v)]
    check(b, *fp4.attention(*x, pool, bt, cu, lens, 0.1))
    check(a, *fp4.attention(*[y[:2] for y in x], pool, bt, [0, 1, 2], lens, 0.1))
    data = fp4.export(f64(rows), bt, cu, [3, 0])
    fp4.import_(data, pool, bt, cu, [3, 0], d)
    assert np.array_equal(buf.cpu().numpy(), data) and np.array_equal(codes.cpu().numpy(), pool)


@pytest.mark.parametrize("option", [(), (("decode_ranges", 7),), (("decode_ranges", 100),), (("decode_parts", 2),)], ids=str)
def test_hundreds_of_requests(option):
    """More requests than a wavefront has lanes, most of them without a cached token in runs: the ranges' look-up takes several to a lane."""
    rng = np.random.default_rng(305)
    hq, hkv, d = 4, 2, 64
    lens = [0] * 90 + [1] * 10 + [int(x) for x in rng.integers(0, 70, size=100)] + [0] * 50 + [400, 0, 0, 33]
    pool, bt = cache(rng, lens, hkv, d, extra=1)
    h = tetri.Tetri(hq, hkv, d, 64, len(pool), bt.shape[1], 8)
    for key, value in option:
        h.tetri_set_option(key, value)
    B = len(lens)
    q, k, v = bf16(rng, B, hq, d), bf16(rng, B, hkv, d), bf16(rng, B, hkv, d)
    out, d_pool = torch.full((B, hq, d), 7.0, dtype=torch.bfloat16, device=DEV), dev(pool)
    h.tetri_decode_attn_fp4(dev(q), dev(k), dev(v), d_pool, dev(bt), dev(np.array(lens, dtype=np.int32)), B, max(lens), d ** -0.5, 1, out)
    torch.cuda.synchronize()
    check(out, *fp4.attention(f64(q), f64(k), f64(v), pool, bt, np.arange(B + 1), lens, d ** -0.5))
    fp4.append(f64(k), f64(v), pool, bt, np.arange(B + 1), lens)
    assert np.array_equal(d_pool.cpu().numpy(), pool)


def test_pages_past_32_bits():
    """A pool of 4.6 GB whose last pages are used: decode, both prefill kernels and the transfers find them."""
    rng = np.random.default_rng(306)
    hq, hkv, d, lens = 16, 8, 128, [75, 20]
    small, bt = cache(rng, lens, hkv, d, extra=40)
    pages = (9 << 29) // (2 * hkv * fp4.slab_bytes(d)) + 1
    assert pages * 2 * hkv * fp4.slab_bytes(d) > 1 << 32
    shift = pages - len(small)
    pool = torch.zeros((pages, 2, hkv, fp4.slab_bytes(d)), dtype=torch.uint8, device=DEV)
    pool[shift:] = dev(small)
    high = dev(bt + shift)
    q, k, v = bf16(rng, 64, hq, d), bf16(rng, 64, hkv, d), bf16(rng, 64, hkv, d)
    x, cu = [f64(y) for y in (q, k, v)], np.array([0, 30, 50], dtype=np.int32)
    d_lens = dev(np.array(lens, dtype=np.int32))
    h = tetri.Tetri(hq, hkv, d, 64, pages, bt.shape[1], 8)
    for variant in (2, 3):
        h.tetri_set_option("attn_variant", variant)
        pool[shift:] = dev(small)
        out = torch.zeros((64, hq, d), dtype=torch.bfloat16, device=DEV)
        h.tetri_chunk_prefill_attn_fp4(dev(q), dev(k), dev(v), pool, high, dev(cu), d_lens, 2, 0.1, 1, out)
        torch.cuda.synchronize()
        check(out, *fp4.attention(*x, small, bt, cu, lens, 0.1))
        want = small.copy()
        fp4.append(x[1], x[2], want, bt, cu, lens)
        assert np.array_equal(pool[shift:].cpu().numpy(), want)
    for ranges in (0, 3):
        h.tetri_set_option("decode_ranges", ranges)
        pool[shift:] = dev(small)
        out = torch.zeros((2, hq, d), dtype=torch.bfloat16, device=DEV)
        h.tetri_decode_attn_fp4(dev(q[:2]), dev(k[:2]), dev(v[:2]), pool, high, d_lens, 2, 75, 0.1, 1, out)
        torch.cuda.synchronize()
        check(out, *fp4.attention(*[y[:2] for y in x], small, bt, [0, 1, 2], lens, 0.1))
        want = small.copy()
        fp4.append(x[1], x[2], want, bt, [0, 1, 2], lens)
        assert np.array_equal(pool[shift:].cpu().numpy(), want)
    # a buffer past 32 bits: the second request's block begins there, the first one's tokens lie in distinct pages in front
    n = [((1 << 32) // (2 * hkv * (d // 2 + d // 32)) // P + 1) * P, 20]
    cu2 = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    blocks = n[0] // P
    wide = torch.zeros((2, blocks), dtype=torch.int32, device=DEV)
    wide[0] = torch.randperm(blocks, device=DEV)
    wide[1, :2] = high[1, :2]
    buf = torch.empty(2 * hkv * (d // 2 + d // 32) * int(cu2[-1]), dtype=torch.uint8, device=DEV)
    assert blocks <= shift and buf.numel() > 1 << 32
    for i in range(0, buf.numel(), 1 << 30):
        buf[i:i + (1 << 30)].random_()
    h2 = tetri.Tetri(hq, hkv, d, 64, pages, blocks, 8)
    h2.tetri_kv_import_fp4(buf, wide, dev(cu2), None, 2, int(cu2[-1]), pool)
    torch.cuda.synchronize()
    size = 2 * hkv * n[0] * d // 2
    codes, exps = buf[:size].view(2 * hkv, n[0], d // 2), buf[size:size + size // 16].view(2 * hkv, n[0], d // 32)
    split = P * d // 2
    for head in range(2 * hkv):
        slabs = pool.view(pages, 2 * hkv, -1)[:, head]
        got = slabs[wide[0].long()]
        assert torch.equal(got[:, :split].reshape(n[0], d // 2), codes[head]) and torch.equal(got[:, split:].reshape(n[0], d // 32), exps[head])
    rest = small.copy()
    fp4.import_(buf[2 * hkv * n[0] * (d // 2 + d // 32):].cpu().numpy(), rest, bt[1:], np.array([0, 20]), None, d)
    assert np.array_equal(pool.view(pages, 2 * hkv, -1)[high[1, 0].long()].cpu().numpy(), rest[bt[1, 0]].reshape(2 * hkv, -1))


def test_a_context_of_millions():
    """4194288 cached tokens: keys of zeros in distinct pages but for three tokens, at the first, the last and a middle place, that take all of the weight in turn."""
    hq, hkv, d = 2, 1, 128
    L, blocks = (1 << 22) - P, 1 << 18
    pool = torch.zeros((blocks, 2, hkv, fp4.slab_bytes(d)), dtype=torch.uint8, device=DEV)
    perm = torch.randperm(blocks, device=DEV).int()
    rng = np.random.default_rng(307)
    places = [0, 2097151, L - 1]
    rows = [rng.standard_normal((1, d)) for _ in places]
    for i, at in enumerate(places):
        page = int(perm[at // P])
        one = pool[page:page + 1].cpu().numpy()
        key = np.zeros((1, d))
        key[0, i] = 6.0
        fp4.store(one, 0, at % P, key, rows[i])
        pool[page] = dev(one[0])
    h = tetri.Tetri(hq, hkv, d, 64, blocks, blocks, 8)
    k, v = torch.zeros((1, 1, d), dtype=torch.bfloat16), torch.zeros((1, 1, d), dtype=torch.bfloat16)
    for ranges in (0, 50):
        h.tetri_set_option("decode_ranges", ranges)
        for i in range(3):
            q = torch.zeros((1, hq, d), dtype=torch.bfloat16)
            q[0, :, i] = 16.0                                # a score of 96 and e^96 against 4 million keys of e^0
            out = torch.zeros((1, hq, d), dtype=torch.bfloat16, device=DEV)
            h.tetri_decode_attn_fp4(dev(q), dev(k), dev(v), pool, perm[None].contiguous(), dev(np.array([L], dtype=np.int32)), 1, L, 1.0, 0, out)
            torch.cuda.synchronize()
            ref = fp4.dequantize(*fp4.quantize(rows[i]))
            # one rounding of the output, one of the weights' sum's factor in 32 bits
            assert (np.abs(out.cpu().float().numpy()[0] - ref) <= (STEP + 2.0 ** -20) * np.abs(ref) + 1e-30).all()


@pytest.mark.parametrize("variant", [0, 2, 3])
def test_prefill_with_keys_that_are_not_numbers(variant):
    """A cached value's group under an exponent of 255 reaches its 32 elements of that head's rows alone; a cached key's, that head's rows; a row of Q, its own."""
    rng = np.random.default_rng(308)
    hq, hkv, d, ctx = 8, 2, 128, [70, 40]
    pool, bt = cache(rng, ctx, hkv, d)
    cu = np.array([0, 33, 60], dtype=np.int32)
    q, k, v = bf16(rng, 64, hq, d), bf16(rng, 64, hkv, d), bf16(rng, 64, hkv, d)
    h = tetri.Tetri(hq, hkv, d, 64, len(pool), bt.shape[1], 8)
    h.tetri_set_option("attn_variant", variant)

    def run(q, pool):
        out = torch.zeros((64, hq, d), dtype=torch.bfloat16, device=DEV)
        h.tetri_chunk_prefill_attn_fp4(dev(q), dev(k), dev(v), dev(pool), dev(bt), dev(cu), dev(np.array(ctx, dtype=np.int32)), 2, 0.1, 0, out)
        torch.cuda.synchronize()
        return out.cpu()
    good = run(q, pool)
    assert not torch.isnan(good).any()
    want = torch.zeros(good.shape, dtype=torch.bool)
    bad = pool.copy()
    bad[bt[0, 0], 1, 1, P * d // 2 + 3 * 4 + 2] = 255
    want[:33, 4:, 64:96] = True
    bad_k = pool.copy()
    bad_k[bt[1, 2], 0, 0, P * d // 2 + 5 * 4] = 255
    want_k = torch.zeros_like(want)
    want_k[33:60, :4] = True
    bad_q, want_q = q.clone(), torch.zeros_like(want)
    bad_q[40, 5, 7] = float("nan")
    want_q[40, 5] = True
    for x, y, nan in ((q, bad, want), (q, bad_k, want_k)):
        out = run(x, y)
        assert torch.equal(torch.isnan(out), nan) and torch.equal(out[~nan].view(torch.int16), good[~nan].view(torch.int16))
    # (rows of a tile may share the moments at which their maxima are raised: not the same bits)
    out = run(bad_q, pool)
    ref, spread = fp4.attention(f64(q), f64(k), f64(v), pool, bt, cu, ctx, 0.1)
    assert torch.equal(torch.isnan(out), want_q)
    check(out[~want_q], ref[~want_q.numpy()], spread[~want_q.numpy()])
