"""Measured work of a KV cache held in 4 bits, and of the step that makes queries and keys ready for it, with their plain forms.

The cache is in the OCP microscaling format MXFP4: 32 neighbouring values of a row of K or V share a power of two, each of them
is an E2M1 code of 4 bits.  A (page, K or V, kv head) takes 16 rows of head_dim / 2 bytes of codes (the even element in the low
half of a byte), then 16 rows of head_dim / 32 bytes, the exponents of the shared powers plus 127.  Five kinds of case, each one
call of a serving program:
  rope     RMS norm of every head of q and k and the rotation by position, out of the rows of a fused projection
  prefill  a chunk's attention over such a cache, its own rows cached in codes in the same call or not
  decode   a decode iteration of a batch over such a cache, likewise
  export   requests' tokens from a 16-bit pool into a dense buffer of codes
  import   such a buffer into the pages of a pool of codes
Head shapes, chunk sizes and lengths are those of the package's synthetic workloads and of its other benchmark cases.
Queries, keys and values are N(0, 1), so that scores are O(1) as in a model; pages lie at random places.
Pools and buffers of codes are returned as the bytes they are, which are the same wherever the values they stand for are.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
PAGE = 16
GROUP = 32
EPS = 1e-6

# (query heads, kv heads, head dim)
HEADS = {"4x64": (4, 4, 64), "40x128": (40, 40, 128), "32/8x128": (32, 8, 128), "8/2x128": (8, 2, 128),
         "6/2x64": (6, 2, 64), "32/1x128": (32, 1, 128)}


def _rope(heads, rows, where, seed, axes=1, rot=0, norm=True, adjacent=False, turns=False, base=10000.0, far=0, fused=True):
    """`rows` tokens.  where "chunk": of a chunk's segments, by its metadata; "given": positions from an array, axes of them.
    rot: values of a head that turn (0: all).  turns: the axes take turns at the frequencies, otherwise they have a run each.
    far: where the positions begin.  fused: the rows lie in a projection of q, k and v, otherwise by themselves."""
    return {"kind": "rope", "heads": heads, "rows": rows, "where": where, "lens_seed": seed, "axes": axes, "rot": rot,
            "norm": norm, "adjacent": adjacent, "turns": turns, "base": base, "far": far, "fused": fused}


def _prefill(heads, chunk, segs, lo, hi, seed, append):
    """A chunk of `segs` segments whose requests have lo..hi tokens cached."""
    return {"kind": "prefill", "heads": heads, "chunk": chunk, "n": segs, "lo": lo, "hi": hi, "lens": "uniform",
            "lens_seed": seed, "append": append}


def _decode(heads, lens, n, lo, hi, seed, append):
    return {"kind": "decode", "heads": heads, "lens": lens, "n": n, "lo": lo, "hi": hi, "lens_seed": seed, "append": append}


def _move(kind, heads, lens, n, lo, hi, seed, first=0):
    """n requests of lo..hi tokens; first: tokens in front of the ones that move."""
    return {"kind": kind, "heads": heads, "lens": lens, "n": n, "lo": lo, "hi": hi, "lens_seed": seed, "first": first}


def listed():
    return [
        # one user's next token, far into a long conversation: the cost is latency
        dict(_rope("40x128", 1, "given", 1, base=1e6, far=100003), name="rope-13b-one"),
        # a chunk of prompts on its way into attention: positions follow from the chunk's metadata
        dict(_rope("40x128", 512, "chunk", 2, norm=False), name="rope-13b-chunk"),
        # throughput serving of a grouped-query model: images and text in one large batch of rows, three axes
        dict(_rope("32/8x128", 8192, "given", 3, axes=3, base=1e6), name="rope-gqa-axes-8k"),
        # prompts packed into a chunk behind ragged contexts, their rows cached as well
        dict(_prefill("32/8x128", 512, 7, 0, 3000, 4, True), name="prefill-gqa-ragged"),
        # a large chunk behind a long context
        dict(_prefill("32/8x128", 2048, 1, 14336, 14336, 5, False), name="prefill-gqa-large"),
        # one user: a single request's next token
        dict(_decode("40x128", "uniform", 1, 1000, 1000, 6, True), name="decode-13b-one"),
        # an ordinary decode batch, every request with the same context
        dict(_decode("40x128", "uniform", 64, 2048, 2048, 7, False), name="decode-13b-64x2k"),
        # a mixed decode batch of a grouped-query model: contexts from tens to thousands of tokens
        dict(_decode("32/8x128", "log", 48, 16, 8192, 8, True), name="decode-gqa-ragged"),
        # chunk-level transfer: the tokens of one chunk
        dict(_move("export", "40x128", "uniform", 1, 512, 512, 9, 1024), name="export-13b-chunk"),
        # request-level transfer of a batch of ragged prompts
        dict(_move("export", "40x128", "uniform", 16, 51, 2048, 10), name="export-13b-ragged"),
        # ... and both where they arrive
        dict(_move("import", "40x128", "uniform", 1, 512, 512, 11, 1024), name="import-13b-chunk"),
        dict(_move("import", "32/8x128", "log", 24, 100, 16384, 12), name="import-gqa-ragged"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "prefill", "decode", "decode", "export", "import"])
    seed = rng.randrange(1 << 20)
    heads = rng.choice(["40x128", "40x128", "32/8x128", "32/8x128", "8/2x128", "4x64", "6/2x64", "32/1x128"])
    hq, hkv, d = HEADS[heads]
    if kind == "rope":
        where = rng.choice(["given", "chunk"])
        axes = 1 if where == "chunk" else rng.choice([1, 2, 3])
        rows = _log_int(rng, 1, 8192 * 40 // max(40, hq + hkv))
        return _rope(heads, rows, where, seed, axes, rng.choice([0, 0, d // 2, 16]), rng.random() < 0.6, rng.random() < 0.3,
                     rng.random() < 0.5, rng.choice([10000.0, 500000.0, 1e6]), rng.choice([0, 0, 5000, 1000003]), rng.random() < 0.7)
    if kind == "prefill":
        chunk = rng.choice([64, 100, 128, 256, 384, 512, 512, 512, 1024, 2048])
        segs = rng.choice([1, 1, 2, _log_int(rng, 1, min(24, max(1, chunk // 4)))])
        # at most the scores of the largest listed case
        hi = _log_int(rng, 1, max(1, min(14336, 1_000_000_000 // (hq * chunk) - chunk)))
        lo = hi if segs == 1 else rng.choice([0, hi // 10])
        return _prefill(heads, chunk, segs, lo, hi, seed, rng.random() < 0.5)
    n = _log_int(rng, 1, 256)
    # the batch's values stay as many as those of the largest listed case
    hi = _log_int(rng, 32, max(64, min(32768, 670_000_000 // (hkv * d * n))))
    if kind != "decode":
        hi = max(64, min(hi, 90_000_000 // (hkv * d * n)))
    how = rng.choice(["same", "uniform", "log"])
    lo = hi if how == "same" else max(1, hi // 20)
    lens = "log" if how == "log" else "uniform"
    if kind == "decode":
        return _decode(heads, lens, n, lo, hi, seed, rng.random() < 0.5)
    return _move(kind, heads, lens, n, lo, hi, seed, rng.choice([0, 0, 7, 256]))


def _lens(case):
    """Tokens of the case's requests: cached ones, or those that move."""
    rng = np.random.default_rng(case["lens_seed"])
    n, lo, hi = case["n"], case["lo"], case["hi"]
    if case["lens"] == "log":
        return [int(round(float(np.exp(x)))) for x in rng.uniform(math.log(lo), math.log(hi), size=n)]
    return [int(x) for x in rng.integers(lo, hi, size=n, endpoint=True)]


def _segments(case, rows, segs):
    """Rows of every segment of a chunk: a random division of it."""
    rng = np.random.default_rng([case["lens_seed"], 1])
    if segs == 1:
        return [rows]
    cuts = np.sort(rng.choice(np.arange(1, rows), size=segs, replace=False))
    return [int(x) for x in np.diff(np.concatenate([[0], cuts]))]      # (the rows behind the last cut are padding)


def _rope_segments(case):
    """... of a rope case: up to 12 segments and some tokens cached in front of each."""
    rng = np.random.default_rng([case["lens_seed"], 2])
    segs = max(1, min(12, case["rows"] // 8))
    return _segments(case, case["rows"], segs), [int(x) for x in case["far"] + rng.integers(0, 3000, size=segs)]


def _values(gen, *shape):
    return torch.randn(shape, dtype=torch.bfloat16, device=DEV, generator=gen)


def _slab(d):
    """Bytes of a (page, K or V, kv head)."""
    return PAGE * (d // 2 + d // GROUP)


def _table(rng, tokens):
    """Random page lists that cover the requests' tokens, and the size of the pool they lie in."""
    need = [-(-n // PAGE) for n in tokens]
    pages = sum(need) + sum(need) // 8 + 1
    perm = rng.permutation(pages).astype(np.int32)
    bt = np.zeros((len(need), max(1, max(need))), dtype=np.int32)
    at = 0
    for r, n in enumerate(need):
        bt[r, :n] = perm[at:at + n]
        at += n
    return bt, pages


def _code_pool(gen, pages, hkv, d):
    """A pool of the codes of N(0, 1) values."""
    pool = torch.empty((pages, 2, hkv, _slab(d)), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 25) // (2 * hkv * PAGE * d))
    for at in range(0, pages, step):
        codes, scales = _quantise(_values(gen, min(step, pages - at), 2, hkv, PAGE, d))
        pool[at:at + step, ..., :PAGE * d // 2] = codes.flatten(-2)
        pool[at:at + step, ..., PAGE * d // 2:] = scales.flatten(-2)
    return pool


def _positions(case, rng):
    """[axes, rows]: runs of text, whose position is the same on all axes, and between them pictures, a grid each."""
    rows, axes = case["rows"], case["axes"]
    if axes == 1:
        return (case["far"] + rng.integers(0, 4096, size=(1, rows))).astype(np.int32)
    pos = np.zeros((axes, rows), dtype=np.int64)
    at, p = 0, case["far"]
    while at < rows:
        n = min(rows - at, int(rng.integers(1, 400)))
        pos[:, at:at + n] = p + np.arange(n)
        at, p = at + n, p + n
        w, hgt = int(rng.integers(4, 40)), int(rng.integers(4, 40))
        n = min(rows - at, w * hgt)
        i = np.arange(n)
        grid = [np.zeros_like(i), i // w, i % w][-axes:]
        for a in range(axes):
            pos[a, at:at + n] = p + grid[a]
        at, p = at + n, p + max(w, hgt)
    return pos.astype(np.int32)


def _frequencies(case):
    """Radians per position of every pair, as 32-bit numbers, and the axis whose position turns it."""
    d = HEADS[case["heads"]][2]
    rot = case["rot"] or d
    half, axes = rot // 2, case["axes"]
    freq = (case["base"] ** (-np.arange(half, dtype=np.float64) / half)).astype(np.float32)
    i = np.arange(half)
    return rot, freq, (i % axes if case["turns"] else i * axes // half).astype(np.uint8)


def _prepare_rope(case, rng, gen):
    hq, hkv, d = HEADS[case["heads"]]
    rows, width = case["rows"], (hq + 2 * hkv) * d
    s = {"case": case}
    if case["fused"]:
        x = _values(gen, rows, width)
        s["q"], s["k"] = x[:, :hq * d], x[:, hq * d:(hq + hkv) * d]
    else:
        s["q"], s["k"] = _values(gen, rows, hq * d), _values(gen, rows, hkv * d)
    s["qw"] = s["kw"] = None
    if case["norm"]:
        s["qw"], s["kw"] = [(1.0 + 0.2 * torch.randn(d, device=DEV, generator=gen)).bfloat16() for _ in range(2)]
    s["cu"] = s["ctx"] = s["pos"] = None
    s["segs"] = 0
    if case["where"] == "chunk":
        parts, ctx = _rope_segments(case)
        s["cu"] = torch.from_numpy(np.concatenate([[0], np.cumsum(parts)]).astype(np.int32)).to(DEV)
        s["ctx"] = torch.tensor(ctx, dtype=torch.int32, device=DEV)
        s["segs"] = len(parts)
    else:
        s["pos"] = torch.from_numpy(_positions(case, rng)).to(DEV)
    s["q_out"] = torch.zeros((rows, hq, d), dtype=torch.bfloat16, device=DEV)
    s["k_out"] = torch.zeros((rows, hkv, d), dtype=torch.bfloat16, device=DEV)
    rot, freq, axis = _frequencies(case)
    s["freq"], s["axis"] = torch.from_numpy(freq).to(DEV), torch.from_numpy(axis).to(DEV).long()
    if own:
        from paper_2401_11181_amd import tetri
        s["h"] = tetri.Tetri(hq, hkv, d, max(rows, 16), 16, 16, 16)
        s["rope"] = tetri.Rope(freq, axis=axis, num_axes=case["axes"], adjacent=case["adjacent"])
    return s


def prepare(case, seed):
    rng = np.random.default_rng([seed, 1])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    hq, hkv, d = HEADS[case["heads"]]
    kind = case["kind"]
    if kind == "rope":
        return _prepare_rope(case, rng, gen)
    lens = _lens(case)
    moves = kind in ("export", "import")
    rows = _segments(case, case["chunk"], case["n"]) if kind == "prefill" else [case["first"] if moves else 1] * len(lens)
    bt, pages = _table(rng, [n + m for n, m in zip(lens, rows)])
    s = {"case": case, "n": len(lens), "max_ctx": max(lens), "total": sum(lens), "scale": 1.0 / math.sqrt(d),
         "bt": torch.from_numpy(bt).to(DEV), "ctx": torch.tensor(lens, dtype=torch.int32, device=DEV)}
    if kind == "export":
        s["pool"] = _values(gen, pages, 2, hkv, PAGE, d)
    else:
        s["pool"] = _code_pool(gen, pages, hkv, d)
    if moves:
        s["cu"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).to(DEV)
        s["first"] = torch.full((len(lens),), case["first"], dtype=torch.int32, device=DEV)
        size = 2 * hkv * (d // 2 + d // GROUP) * s["total"]
        if kind == "export":
            s["buf"] = torch.zeros(size, dtype=torch.uint8, device=DEV)
        else:
            s["buf"] = torch.randint(0, 256, (size,), dtype=torch.uint8, device=DEV, generator=gen)
    elif kind == "prefill":
        s["cu"] = torch.from_numpy(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)).to(DEV)
        s["most_rows"] = max(rows)
        c = case["chunk"]
        s["q"], s["k"], s["v"] = _values(gen, c, hq, d), _values(gen, c, hkv, d), _values(gen, c, hkv, d)
        s["out"] = torch.zeros_like(s["q"])
    else:
        b = len(lens)
        s["q"], s["k"], s["v"] = _values(gen, b, hq, d), _values(gen, b, hkv, d), _values(gen, b, hkv, d)
        s["out"] = torch.zeros_like(s["q"])
    if own:
        from paper_2401_11181_amd import tetri
        chunk = case["chunk"] if kind == "prefill" else 64
        s["h"] = tetri.Tetri(hq, hkv, d, chunk, pages, bt.shape[1], min(chunk, 64), page_size=PAGE)
    return s


# ---- the plain forms

def _quantise(x):
    """Codes and scales of rows of values [..., D]: two codes to a byte [..., D / 2], a scale's exponent plus 127 [..., D / 32]."""
    y = x.float().unflatten(-1, (-1, GROUP))
    top = y.abs().amax(-1, keepdim=True)
    usable = torch.isfinite(top)
    power = torch.frexp(torch.where(usable, top, 1.0))[1] - 3           # floor(log2 top) - 2: 6 * 2^power or a little less is top
    power = torch.where(top == 0, -127, power.clamp(min=-127))
    size = torch.where(usable, torch.ldexp(y.abs(), -power), 0.0)
    # the nearest of 0 0.5 1 1.5 2 3 4 6, of two equally near ones that with an even code
    code = ((size > 0.25).byte() + (size >= 0.75) + (size > 1.25) + (size >= 1.75) + (size > 2.5) + (size >= 3.5) + (size > 5.0))
    code = torch.where(usable, code + 8 * torch.signbit(y), 0).to(torch.uint8).flatten(-2)
    scale = torch.where(usable, power + 127, 255).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale.squeeze(-1)


def _read(pool, d):
    """The values of slabs [..., slab bytes]: [..., PAGE, D] as 32-bit numbers."""
    codes = pool[..., :PAGE * d // 2].unflatten(-1, (PAGE, d // 2))
    scales = pool[..., PAGE * d // 2:].unflatten(-1, (PAGE, d // GROUP))
    size = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    size = torch.cat([size, -size])
    x = torch.stack([size[(codes & 15).long()], size[(codes >> 4).long()]], -1).flatten(-2)
    power = torch.where(scales == 255, math.nan, torch.exp2(scales.float() - 127))
    return (x.unflatten(-1, (-1, GROUP)) * power[..., None]).flatten(-2)


def _cached(s, which):
    """[requests, kv heads, table slots, head dim]: what the block table names, K (0) or V (1)."""
    x = _read(s["pool"][:, which][s["bt"].long()], s["q"].shape[-1])     # [B, blocks, Hkv, PAGE, D]
    b, blocks, hkv, _, d = x.shape
    return x.transpose(1, 2).reshape(b, hkv, blocks * PAGE, d)


def _cache_rows(s, page, slot, k, v):
    """Rows k, v [n, Hkv, D] go to the given pages and slots in codes."""
    d = k.shape[-1]
    codes, scales = _quantise(torch.stack([k, v], 1))                    # [n, 2, Hkv, ...]
    slabs = s["pool"]
    slabs[..., :PAGE * d // 2].unflatten(-1, (PAGE, d // 2))[page, :, :, slot] = codes
    slabs[..., PAGE * d // 2:].unflatten(-1, (PAGE, d // GROUP))[page, :, :, slot] = scales


def _attention_outputs(s):
    return {"out": s["out"], "pool": s["pool"]} if s["case"]["append"] else {"out": s["out"]}


def _plain_rope(s):
    case = s["case"]
    hq, hkv, d = HEADS[case["heads"]]
    rows = case["rows"]
    real = rows
    if case["where"] == "chunk":
        row = torch.arange(rows, device=DEV)
        seg = torch.searchsorted(s["cu"][1:].contiguous(), row.int(), right=True)
        real = row < s["cu"][-1]
        seg = seg.clamp(max=s["segs"] - 1)
        pos = (s["ctx"].long()[seg] + row - s["cu"].long()[seg])[None]
    else:
        pos = s["pos"].long()
    angle = pos.double()[s["axis"]].T * s["freq"].double()               # [rows, pairs]; 32 bits lose far positions
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    half = s["freq"].numel()
    got = {}
    for name, x, weight, heads in (("q_out", s["q"], s["qw"], hq), ("k_out", s["k"], s["kw"], hkv)):
        x = x.float().view(rows, heads, d)
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
        turning, rest = x[..., :2 * half], x[..., 2 * half:]
        a, b = (turning[..., 0::2], turning[..., 1::2]) if case["adjacent"] else (turning[..., :half], turning[..., half:])
        a, b = a * cos - b * sin, b * cos + a * sin
        turning = torch.stack([a, b], -1).flatten(-2) if case["adjacent"] else torch.cat([a, b], -1)
        x = torch.cat([turning, rest], -1).bfloat16()
        if case["where"] == "chunk":
            x = torch.where(real[:, None, None], x, s[name])
        got[name] = s[name].copy_(x)
    return got


def _plain_prefill(s):
    case = s["case"]
    hq, hkv, d = HEADS[case["heads"]]
    g = hq // hkv
    cu, ctx = s["cu"].long(), s["ctx"].long()
    n_new, first, m = cu[1:] - cu[:-1], cu[:-1], s["most_rows"]
    row = torch.arange(m, device=DEV).expand(len(ctx), m)
    is_row = row < n_new[:, None]
    at = (first[:, None] + row).clamp(max=case["chunk"] - 1)
    width = s["bt"].shape[1] * PAGE
    old = torch.arange(width, device=DEV)
    q = s["q"][at].float().view(-1, m, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(len(ctx), hkv, m * g, d)
    k_new, v_new = s["k"][at].float().transpose(1, 2), s["v"][at].float().transpose(1, 2)
    scores = torch.matmul(q, torch.cat([_cached(s, 0), k_new], 2).transpose(2, 3)).mul_(s["scale"])
    see_old = (old < ctx[:, None])[:, None, :].expand(-1, m, -1)
    see_new = (row[:, None, :] <= row[:, :, None]) & is_row[:, None, :]
    unseen = ~torch.cat([see_old, see_new], 2)[:, None, :, None, :]
    shaped = scores.view(len(ctx), hkv, m, g, -1).masked_fill_(unseen, -math.inf)
    shaped.sub_(shaped.amax(-1, keepdim=True)).exp_()                    # (every row sees its own key, or the first)
    shaped.div_(shaped.sum(-1, keepdim=True))
    values = torch.cat([torch.where((old < ctx[:, None])[:, None, :, None], _cached(s, 1), 0.0), v_new], 2)
    out = torch.matmul(scores, values).view(len(ctx), hkv, m, g, d).permute(0, 2, 1, 3, 4).reshape(len(ctx), m, hq, d)
    s["out"].zero_()
    s["out"][at[is_row]] = out[is_row].bfloat16()
    if case["append"]:
        pos = (ctx[:, None] + row)[is_row]
        page = s["bt"].long()[torch.arange(len(ctx), device=DEV)[:, None].expand_as(row)[is_row], pos // PAGE]
        _cache_rows(s, page, pos % PAGE, s["k"][at[is_row]], s["v"][at[is_row]])
    return _attention_outputs(s)


def _plain_decode(s):
    case = s["case"]
    hq, hkv, d = HEADS[case["heads"]]
    ctx, bt = s["ctx"].long(), s["bt"].long()
    b, width = len(ctx), bt.shape[1] * PAGE
    dead = (torch.arange(width, device=DEV) >= ctx[:, None])[:, None]
    q = s["q"].float().view(b, hkv, hq // hkv, d)
    own_score = (q * s["k"].float()[:, :, None]).sum(-1, keepdim=True)
    scores = torch.cat([torch.matmul(q, _cached(s, 0).transpose(2, 3)), own_score], 3).mul_(s["scale"])
    scores[..., :width].masked_fill_(dead[:, :, None], -math.inf)
    scores = (scores - scores.amax(-1, keepdim=True)).exp_()
    p = scores / scores.sum(-1, keepdim=True)
    values = torch.where(dead[..., None], 0.0, _cached(s, 1))
    out = torch.matmul(p[..., :width], values) + p[..., width:] * s["v"].float()[:, :, None]
    s["out"].copy_(out.view(b, hq, d))
    if case["append"]:
        _cache_rows(s, bt.gather(1, ctx[:, None] // PAGE)[:, 0], ctx % PAGE, s["k"], s["v"])
    return _attention_outputs(s)


def _moved(s):
    """Pages and slots of the tokens that move, in the buffer's order, and the request of each."""
    cu, case = s["cu"].long(), s["case"]
    token = torch.arange(s["total"], device=DEV)
    req = torch.searchsorted(cu[1:].contiguous(), token, right=True)
    pos = s["first"].long()[req] + token - cu[req]
    return s["bt"].long()[req, pos // PAGE], pos % PAGE, req, token - cu[req]


def _places(s, req, j, row_bytes, skip):
    """Bytes of the buffer that hold rows of row_bytes: token j of request req, [tokens, 2 * Hkv, row_bytes].  skip: row bytes
    of what lies in front of them in a request's block."""
    hkv, d = HEADS[s["case"]["heads"]][1:]
    cu = s["cu"].long()
    n = (cu[1:] - cu[:-1])[req]
    begin = 2 * hkv * ((d // 2 + d // GROUP) * cu[req] + skip * n)
    row = begin[:, None] + (torch.arange(2 * hkv, device=DEV) * n[:, None] + j[:, None]) * row_bytes
    return row[..., None] + torch.arange(row_bytes, device=DEV)


def _plain_export(s):
    page, slot, req, j = _moved(s)
    d = s["pool"].shape[-1]
    codes, scales = _quantise(s["pool"][page, :, :, slot])               # [tokens, 2, Hkv, ...]
    s["buf"][_places(s, req, j, d // 2, 0)] = codes.flatten(1, 2)
    s["buf"][_places(s, req, j, d // GROUP, d // 2)] = scales.flatten(1, 2)
    return {"buf": s["buf"]}


def _plain_import(s):
    page, slot, req, j = _moved(s)
    hkv, d = HEADS[s["case"]["heads"]][1:]
    codes = s["buf"][_places(s, req, j, d // 2, 0)].unflatten(1, (2, hkv))
    scales = s["buf"][_places(s, req, j, d // GROUP, d // 2)].unflatten(1, (2, hkv))
    s["pool"][..., :PAGE * d // 2].unflatten(-1, (PAGE, d // 2))[page, :, :, slot] = codes
    s["pool"][..., PAGE * d // 2:].unflatten(-1, (PAGE, d // GROUP))[page, :, :, slot] = scales
    return {"pool": s["pool"]}


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        return {"rope": _plain_rope, "prefill": _plain_prefill, "decode": _plain_decode, "export": _plain_export,
                "import": _plain_import}[kind](s)
    h = s["h"]
    if kind == "rope":
        h.tetri_qk_norm_rope(s["q"], s["q"].stride(0), s["k"], s["k"].stride(0), s["qw"], s["kw"], EPS, s["rope"], s["pos"],
                             s["cu"], s["ctx"], s["segs"], case["rows"], s["q_out"], s["k_out"])
        return {"q_out": s["q_out"], "k_out": s["k_out"]}
    if kind == "prefill":
        h.tetri_chunk_prefill_attn_fp4(s["q"], s["k"], s["v"], s["pool"], s["bt"], s["cu"], s["ctx"], s["n"], s["scale"],
                                       int(case["append"]), s["out"])
        return _attention_outputs(s)
    if kind == "decode":
        h.tetri_decode_attn_fp4(s["q"], s["k"], s["v"], s["pool"], s["bt"], s["ctx"], s["n"], s["max_ctx"], s["scale"],
                                int(case["append"]), s["out"])
        return _attention_outputs(s)
    if kind == "export":
        h.tetri_kv_export_fp4(s["pool"], s["bt"], s["cu"], s["first"], s["n"], s["total"], s["buf"])
        return {"buf": s["buf"]}
    h.tetri_kv_import_fp4(s["buf"], s["bt"], s["cu"], s["first"], s["n"], s["total"], s["pool"])
    return {"pool": s["pool"]}


def work(case):
    hq, hkv, d = HEADS[case["heads"]]
    row = d // 2 + d // GROUP                                            # bytes of a row of codes
    if case["kind"] == "rope":
        rows = sum(_rope_segments(case)[0]) if case["where"] == "chunk" else case["rows"]
        size = rows * ((hq + hkv) * d * 4 + (4 * case["axes"] if case["where"] == "given" else 0))
        return {"bytes": size, "flops": rows * (hq + hkv) * (3.0 * (case["rot"] or d) + (4.0 * d if case["norm"] else 0.0))}
    lens = _lens(case)
    total = sum(lens)
    if case["kind"] in ("export", "import"):
        return {"bytes": total * 2 * hkv * (row + (2 * d if case["kind"] == "export" else row)), "flops": 0}
    if case["kind"] == "prefill":
        rows = _segments(case, case["chunk"], case["n"])
        # what is cached, the chunk's rows, what comes out (the padding rows of it too) and what is cached of them
        size = total * hkv * 2 * row + sum(rows) * (2 * hq + 4 * hkv) * d + case["chunk"] * hq * d * 2
        size += sum(rows) * hkv * 2 * row if case["append"] else 0
        return {"bytes": size, "flops": 4.0 * d * hq * sum(n * L + n * (n + 1) // 2 for n, L in zip(rows, lens))}
    new = len(lens) * (4 * hq * d + 4 * hkv * d + (2 * row * hkv if case["append"] else 0))
    return {"bytes": total * hkv * 2 * row + new, "flops": sum(4.0 * d * hq * (n + 1) for n in lens)}


# ---- the definitions in 64 bits

def _rows64(s, r, which, kh, d):
    """K (0) or V (1) of the cached tokens of request r and one kv head, [ctx, D]."""
    length = int(s["ctx"][r])
    slab = s["pool"][s["bt"][r, :-(-length // PAGE)].long(), which, kh].long()
    code = slab[:, :PAGE * d // 2].reshape(-1, d // 2)
    code = torch.stack([code % 16, code // 16], 2).reshape(-1, d)
    exponent, fraction = code // 2 % 4, code % 2
    x = torch.where(exponent == 0, fraction / 2.0, (1.0 + fraction / 2.0) * 2.0 ** (exponent - 1).double())
    x = torch.where(code >= 8, -x, x).double()
    power = 2.0 ** (slab[:, PAGE * d // 2:].reshape(-1, d // GROUP).double() - 127.0)
    return (x * power.repeat_interleave(GROUP, 1))[:length]


def _exact_rope(s):
    case = s["case"]
    hq, hkv, d = HEADS[case["heads"]]
    if case["where"] == "chunk":
        parts, ctx = _rope_segments(case)
        pos = torch.cat([torch.arange(c, c + n, dtype=torch.float64, device=DEV) for n, c in zip(parts, ctx)])[None]
    else:
        pos = s["pos"].double()
    rows = pos.shape[1]
    pairs = s["freq"].numel()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos[s["axis"]].T * s["freq"].double())
    got = {}
    for name, x, weight, heads in (("q_out", s["q"], s["qw"], hq), ("k_out", s["k"], s["kw"], hkv)):
        y = x[:rows].double().reshape(rows, heads, d)
        if weight is not None:
            y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + float(np.float32(EPS))) * weight.double()
        y = y.clone()
        first = torch.arange(pairs, device=DEV) * (2 if case["adjacent"] else 1)
        second = first + (1 if case["adjacent"] else pairs)
        z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        got[name] = s[name].double()
        got[name][:rows] = y
    return got


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rope":
        return _exact_rope(s)
    if kind in ("export", "import"):
        return None                              # (bytes)
    hq, hkv, d = HEADS[case["heads"]]
    g = hq // hkv
    scale = float(np.float32(s["scale"]))
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    cu = s["cu"].tolist() if kind == "prefill" else list(range(s["n"] + 1))
    for r in range(s["n"]):
        a, b, length = cu[r], cu[r + 1], int(s["ctx"][r])
        hidden = torch.arange(length + b - a, device=DEV)[None] > length + torch.arange(b - a, device=DEV)[:, None]
        for kh in range(hkv):
            keys = torch.cat([_rows64(s, r, 0, kh, d), s["k"][a:b, kh].double()])
            vals = torch.cat([_rows64(s, r, 1, kh, d), s["v"][a:b, kh].double()])
            for h in range(kh * g, kh * g + g):
                x = (s["q"][a:b, h].double() @ keys.T) * scale
                out[a:b, h] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ vals
    # (the pool has no computed numbers but the codes of the new rows, which are rounded)
    return {"out": out, "pool": None} if case["append"] else {"out": out}
