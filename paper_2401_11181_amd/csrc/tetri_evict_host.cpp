// Host layer of the calls that weigh cached tokens, choose which of them stay and close the cache up (argument checks, launch
// shapes, workspaces).
#include <algorithm>
#include <cmath>

#include "tetri_internal.h"

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

tetri_status check_pointers(tetri_ctx *h, const char *fn, const void *const *ptrs, const char *const *names, int n)
{
    for (int i = 0; i < n; ++i) {
        if (!ptrs[i]) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: %s is null", fn, names[i]);
        if (!aligned16(ptrs[i])) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: %s is not 16-byte aligned", fn, names[i]);
    }
    return TETRI_OK;
}

tetri_status check_device(tetri_ctx *h, const char *fn)
{
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != h->device)
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: the handle was created on device %d, the current device is %d", fn, h->device, dev);
    return TETRI_OK;
}

int64_t most_tokens(const tetri_ctx *h) { return (int64_t)h->cfg.max_blocks_per_seq * h->cfg.page_size; }

tetri_status check_max_ctx(tetri_ctx *h, const char *fn, int32_t max_ctx_len)
{
    if (max_ctx_len < 0 || max_ctx_len > most_tokens(h))
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: max_ctx_len=%d outside 0..%lld", fn, max_ctx_len, (long long)most_tokens(h));
    return TETRI_OK;
}

tetri_status check_reqs(tetri_ctx *h, const char *fn, int32_t num_reqs)
{
    if (num_reqs < 1 || (int64_t)num_reqs * h->cfg.num_kv_heads > (1 << 24))
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: num_reqs=%d outside 1..%d", fn, num_reqs, (1 << 24) / h->cfg.num_kv_heads);
    return TETRI_OK;
}

tetri_status check_segs(tetri_ctx *h, const char *fn, int32_t num_segs, int32_t last_rows)
{
    if (num_segs < 1 || num_segs > h->cfg.max_segs_per_chunk)
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: num_segs=%d outside 1..%d", fn, num_segs, h->cfg.max_segs_per_chunk);
    if (last_rows < 1) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: last_rows=%d is not positive", fn, last_rows);
    return TETRI_OK;
}

tetri_status check_workspace(tetri_ctx *h, const char *fn, const void *workspace, int64_t bytes, int64_t need)
{
    if (!workspace || !aligned16(workspace)) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: workspace is null or not 16-byte aligned", fn);
    if (bytes < need)
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld are needed", fn, (long long)bytes, (long long)need);
    return TETRI_OK;
}

int64_t score_stride(int32_t max_ctx_len) { return ((int64_t)max_ctx_len + 1 + 31) / 32 * 32; }

int64_t decode_bytes(const tetri_ctx *h, int32_t num_reqs, int32_t max_ctx_len)
{
    return (int64_t)num_reqs * h->cfg.num_q_heads * (score_stride(max_ctx_len) + 2) * 4;
}

// How the first pass of weighing a chunk is cut.  Wavefronts of a workgroup that have rows of their own share the keys they read: as many as a
// segment's rows fill, on average, and not so many that workgroups are lacking.  The keys of a row tile are cut in as many parts as
// give every compute unit two workgroups, none of fewer than eight tiles of keys.  (40 heads, 512 rows, no context: 22 us with wavefronts of
// one's own, 27 with four that share; 256 rows behind 8000 tokens: 87 and 80.)  Of several segments each ends in half a row tile on average, and
// workgroups that are more than that begin when the others have ended: 7 segments of up to 3000 tokens over codes, 512 rows, 8 kv heads: 45.4 us with
// 3 parts, 48.7 with the 4 of full tiles.  (With contexts of very different lengths more parts are better: 6 of up to 11668 tokens 86 us instead of
// 99.  Parts of the same length for all segments, and more of them, were not better on the whole.)
struct WeighShape {
    int32_t row_waves, parts;
};
WeighShape weigh_shape(const tetri_ctx *h, int32_t num_segs, int32_t max_ctx_len, int32_t last_rows)
{
    const int64_t g = h->cfg.num_q_heads / h->cfg.num_kv_heads, rows = std::min<int64_t>(h->cfg.chunk_size, (int64_t)num_segs * last_rows) * g;
    const int64_t mean = rows / num_segs, places = 2 * std::max(h->num_cus, 1);
    const int64_t tiles = ((int64_t)max_ctx_len + std::min(h->cfg.chunk_size, last_rows)) / 32 + 2;
    WeighShape w;
    for (w.row_waves = mean >= 512 ? 4 : mean > 64 ? 2 : 1;; w.row_waves /= 2) {
        const int64_t tile = 64 * w.row_waves, wgs = (rows + (tile - 1) * (num_segs + 1) / 2) / tile * h->cfg.num_kv_heads;
        w.parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>({places / wgs, tiles / 8, kWeighParts}));
        if (w.row_waves == 1 || wgs * w.parts >= places * 3 / 4) return w;
    }
}

int64_t weigh_bytes(const tetri_ctx *h, int32_t num_segs, int32_t max_ctx_len, int32_t last_rows)
{
    const int64_t parts = weigh_shape(h, num_segs, max_ctx_len, last_rows).parts;
    return (int64_t)h->cfg.chunk_size * h->cfg.num_q_heads * (parts > 1 ? 8 * parts + 4 : 4);
}

}  // namespace

extern "C" {

int64_t tetri_decode_attn_weights_workspace(tetri_ctx *h, int32_t num_reqs, int32_t max_ctx_len)
{
    const char *fn = "tetri_decode_attn_weights_workspace";
    if (!h) return tetri_fail(nullptr, TETRI_ERR_INVALID_ARG, "%s: null handle", fn);
    tetri_status st = check_reqs(h, fn, num_reqs);
    if (st == TETRI_OK) st = check_max_ctx(h, fn, max_ctx_len);
    return st == TETRI_OK ? decode_bytes(h, num_reqs, max_ctx_len) : st;
}

tetri_status tetri_decode_attn_weights(tetri_ctx *h, const void *q, const void *k_new, const void *v_new, void *kv_pages, float *kv_weights,
                                       const int32_t *block_table, const int32_t *ctx_lens, int32_t num_reqs, int32_t max_ctx_len, float scale,
                                       int32_t append, int32_t fp8, float k_scale, float v_scale, void *workspace, int64_t workspace_bytes, void *out,
                                       void *stream)
{
    const char *fn = "tetri_decode_attn_weights";
    if (!h) return tetri_fail(nullptr, TETRI_ERR_INVALID_ARG, "%s: null handle", fn);
    if ((append != 0 && append != 1) || (fp8 != 0 && fp8 != 1)) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: append and fp8 must be 0 or 1", fn);
    const void *ptrs[] = {kv_weights};
    const char *names[] = {"kv_weights"};
    tetri_status st = check_pointers(h, fn, ptrs, names, 1);
    if (st == TETRI_OK) st = check_reqs(h, fn, num_reqs);
    if (st == TETRI_OK) st = check_max_ctx(h, fn, max_ctx_len);
    if (st == TETRI_OK) st = check_workspace(h, fn, workspace, workspace_bytes, decode_bytes(h, num_reqs, max_ctx_len));
    if (st != TETRI_OK) return st;
    const size_t heads = (size_t)num_reqs * h->cfg.num_q_heads;
    DecodeWeights w;
    w.score_stride = (int32_t)score_stride(max_ctx_len);
    w.max_ctx = max_ctx_len;
    w.scores = static_cast<float *>(workspace);
    w.new_scores = w.scores + heads * w.score_stride;
    w.lse = w.new_scores + heads;
    // The workgroup that finishes a (request, kv head) also adds its weights where that is little work, for one and for all: it saves a launch (one
    // request of 1000 tokens, 40 heads: 11.8 us against 13.5), but that workgroup does it alone, behind everything else (48 requests of up to 8192
    // tokens, 32/8 heads: 69 against 59; 64 of 2048, 40 heads: 457 against 450).
    const bool fused = (int64_t)max_ctx_len * (h->cfg.num_q_heads / h->cfg.num_kv_heads) <= 8192 &&
                       (int64_t)max_ctx_len * num_reqs * h->cfg.num_q_heads <= (1 << 20);
    w.weights_w = fused ? kv_weights : nullptr;
    st = tetri_decode_call(fn, h, q, k_new, v_new, kv_pages, append ? kv_pages : nullptr, block_table, ctx_lens, num_reqs, max_ctx_len, scale, out,
                           stream, fp8 != 0, k_scale, v_scale, &w);
    if (st != TETRI_OK || fused) return st;
    AddWeightsParams p;
    p.scores = w.scores; p.new_scores = fp8 ? w.new_scores : nullptr; p.lse = w.lse;
    p.weights = kv_weights;
    p.bt = block_table; p.ctx = ctx_lens;
    p.B = num_reqs; p.Hq = h->cfg.num_q_heads; p.Hkv = h->cfg.num_kv_heads; p.g = p.Hq / p.Hkv;
    p.max_blocks = h->cfg.max_blocks_per_seq; p.score_stride = w.score_stride; p.max_ctx = max_ctx_len; p.append = append;
    const hipError_t e = tetri_launch_add_weights(p, max_ctx_len, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return tetri_fail(h, TETRI_ERR_HIP, "%s: launch failed: %s", fn, hipGetErrorString(e));
    return TETRI_OK;
}

int64_t tetri_chunk_prefill_weights_workspace(tetri_ctx *h, int32_t num_segs, int32_t max_ctx_len, int32_t last_rows)
{
    const char *fn = "tetri_chunk_prefill_weights_workspace";
    if (!h) return tetri_fail(nullptr, TETRI_ERR_INVALID_ARG, "%s: null handle", fn);
    tetri_status st = check_segs(h, fn, num_segs, last_rows);
    if (st == TETRI_OK) st = check_max_ctx(h, fn, max_ctx_len);
    return st == TETRI_OK ? weigh_bytes(h, num_segs, max_ctx_len, last_rows) : st;
}

tetri_status tetri_chunk_prefill_weights(tetri_ctx *h, const void *q, const void *k_new, const void *kv_pages, float *kv_weights,
                                         const int32_t *block_table, const int32_t *cu, const int32_t *ctx_lens, int32_t num_segs,
                                         int32_t max_ctx_len, int32_t last_rows, float scale, int32_t fp8, float k_scale, void *workspace,
                                         int64_t workspace_bytes, void *stream)
{
    const char *fn = "tetri_chunk_prefill_weights";
    if (!h) return tetri_fail(nullptr, TETRI_ERR_INVALID_ARG, "%s: null handle", fn);
    if (fp8 != 0 && fp8 != 1) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: fp8 must be 0 or 1", fn);
    const void *ptrs[] = {q, k_new, kv_pages, kv_weights};
    const char *names[] = {"q", "k_new", "kv_pages", "kv_weights"};
    tetri_status st = check_pointers(h, fn, ptrs, names, 4);
    if (st != TETRI_OK) return st;
    if (!block_table || !cu || !ctx_lens) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: null metadata pointer", fn);
    if (!std::isfinite(scale)) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: scale is not finite", fn);
    if (fp8 && !(std::isfinite(k_scale) && k_scale > 0.f)) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: k_scale must be positive and finite", fn);
    st = check_segs(h, fn, num_segs, last_rows);
    if (st == TETRI_OK) st = check_max_ctx(h, fn, max_ctx_len);
    if (st == TETRI_OK) st = check_workspace(h, fn, workspace, workspace_bytes, weigh_bytes(h, num_segs, max_ctx_len, last_rows));
    if (st == TETRI_OK) st = check_device(h, fn);
    if (st != TETRI_OK) return st;
    const tetri_config &c = h->cfg;
    WeighParams p;
    p.q = static_cast<const uint16_t *>(q); p.k_new = static_cast<const uint16_t *>(k_new);
    p.pages = static_cast<const uint16_t *>(kv_pages);
    p.weights = kv_weights;
    p.bt = block_table; p.cu = cu; p.ctx = ctx_lens;
    p.S = num_segs; p.C = c.chunk_size; p.Hq = c.num_q_heads; p.Hkv = c.num_kv_heads; p.g = p.Hq / p.Hkv;
    p.max_blocks = c.max_blocks_per_seq; p.max_ctx = max_ctx_len;
    p.last = std::min(last_rows, c.chunk_size);
    const WeighShape shape = weigh_shape(h, num_segs, max_ctx_len, last_rows);
    p.row_waves = shape.row_waves; p.parts = shape.parts;
    p.stats = static_cast<float2 *>(workspace);
    p.lse = static_cast<float *>(workspace) + (p.parts > 1 ? (size_t)2 * p.C * p.Hq * p.parts : 0);
    // 64 keys to a wavefront of the second pass where that still gives nearly every compute unit two workgroups (of several requests the longest is
    // known: the others are taken for half as long on average).  16896 keys of 8 kv heads, 128 query rows each: 33 us in all against 36 with 32 keys;
    // 2048 keys of 40 heads, 512 rows: 45 against 44; 7 segments of up to 3000 tokens over codes, 8 kv heads: 51 against 46.
    p.wide_keys = ((int64_t)max_ctx_len * (num_segs + 1) / 2 + c.chunk_size) / 256 * p.Hkv >= 15 * (int64_t)h->num_cus / 8;
    p.g_magic = p.g <= 1 ? 0u : (uint32_t)((0x100000000ull + p.g - 1) / p.g);
    // (never 0: a masked score is an infinity, which the factor turns into -infinity)
    const auto factor = [&](float of) { return std::copysign(std::fmax(std::fabs(scale) * 1.4426950408889634f * of, 1e-30f), scale); };
    p.c = factor(1.f);
    p.c_codes = factor(fp8 ? k_scale : 1.f);
    const int64_t rows = std::min<int64_t>(p.C, (int64_t)p.S * p.last) * p.g;
    if ((rows / 64 + p.S) * p.parts * p.Hkv > 0x7fffffff || ((int64_t)p.C * p.g + 64) * p.g > 0xffffffffll ||
        (int64_t)p.C * p.Hq * c.head_dim * 2 > 0xffffffffll)
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: too many rows for one launch", fn);
    const hipError_t e = tetri_launch_weigh(c.head_dim, fp8 != 0, p, h->num_cus, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return tetri_fail(h, TETRI_ERR_HIP, "%s: launch failed: %s", fn, hipGetErrorString(e));
    return TETRI_OK;
}

static tetri_status check_budget(tetri_ctx *h, const char *fn, int32_t num_reqs, int32_t keep, int32_t recent)
{
    tetri_status st = check_reqs(h, fn, num_reqs);
    if (st != TETRI_OK) return st;
    if (keep < 1 || keep > most_tokens(h)) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: keep=%d outside 1..%lld", fn, keep, (long long)most_tokens(h));
    if (recent < 0 || recent > keep) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: recent=%d outside 0..keep=%d", fn, recent, keep);
    return TETRI_OK;
}

tetri_status tetri_kv_select(tetri_ctx *h, const float *kv_weights, const int32_t *block_table, const int32_t *ctx_lens, int32_t num_reqs,
                             int32_t max_ctx_len, int32_t keep, int32_t recent, int32_t *slots, int32_t *new_lens, void *stream)
{
    const char *fn = "tetri_kv_select";
    if (!h) return tetri_fail(nullptr, TETRI_ERR_INVALID_ARG, "%s: null handle", fn);
    const void *ptrs[] = {kv_weights, slots};
    const char *names[] = {"kv_weights", "slots"};
    tetri_status st = check_pointers(h, fn, ptrs, names, 2);
    if (st != TETRI_OK) return st;
    if (!block_table || !ctx_lens || !new_lens) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: null metadata pointer", fn);
    if (new_lens == ctx_lens) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: new_lens is ctx_lens", fn);
    st = check_budget(h, fn, num_reqs, keep, recent);
    if (st == TETRI_OK) st = check_max_ctx(h, fn, max_ctx_len);
    if (st != TETRI_OK) return st;
    if (max_ctx_len > kSelectMost)
        return tetri_fail(h, TETRI_ERR_UNSUPPORTED, "%s: max_ctx_len=%d, at most %d tokens are chosen from", fn, max_ctx_len, kSelectMost);
    st = check_device(h, fn);
    if (st != TETRI_OK) return st;
    SelectParams p = {kv_weights, block_table, ctx_lens, slots, new_lens, num_reqs, h->cfg.num_kv_heads, h->cfg.max_blocks_per_seq, max_ctx_len, keep, recent};
    const hipError_t e = tetri_launch_select(p, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return tetri_fail(h, TETRI_ERR_HIP, "%s: launch failed: %s", fn, hipGetErrorString(e));
    return TETRI_OK;
}

tetri_status tetri_kv_compact(tetri_ctx *h, const int32_t *slots, const int32_t *block_table, const int32_t *ctx_lens, int32_t num_reqs, int32_t keep,
                              int32_t recent, void *kv_pages, float *kv_weights, int32_t fp8, void *stream)
{
    const char *fn = "tetri_kv_compact";
    if (!h) return tetri_fail(nullptr, TETRI_ERR_INVALID_ARG, "%s: null handle", fn);
    if (fp8 != 0 && fp8 != 1) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: fp8 must be 0 or 1", fn);
    const void *ptrs[] = {slots, kv_pages, kv_weights};
    const char *names[] = {"slots", "kv_pages", "kv_weights"};
    tetri_status st = check_pointers(h, fn, ptrs, names, 3);
    if (st != TETRI_OK) return st;
    if (!block_table || !ctx_lens) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: null metadata pointer", fn);
    st = check_budget(h, fn, num_reqs, keep, recent);
    if (st == TETRI_OK) st = check_device(h, fn);
    if (st != TETRI_OK) return st;
    CompactParams p = {slots, block_table, ctx_lens, static_cast<char *>(kv_pages), kv_weights, num_reqs, h->cfg.num_kv_heads, h->cfg.max_blocks_per_seq, keep, recent};
    // (a workgroup has 256 slots of one kv head)
    if ((int64_t)num_reqs * h->cfg.num_kv_heads * (keep / 256 + 3) > 0x7fffffff)
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: too many tokens for one launch", fn);
    const hipError_t e = tetri_launch_compact(h->cfg.head_dim * (fp8 ? 1 : 2), p, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return tetri_fail(h, TETRI_ERR_HIP, "%s: launch failed: %s", fn, hipGetErrorString(e));
    return TETRI_OK;
}

}  // extern "C"
