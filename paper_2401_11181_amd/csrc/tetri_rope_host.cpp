// Host layer of the norm and rotation of queries and keys.
#include <algorithm>
#include <cmath>

#include "tetri_internal.h"

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

extern "C" {

tetri_status tetri_qk_norm_rope(tetri_ctx *h, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *q_weight,
                                const void *k_weight, float eps, const tetri_rope *rope, const int32_t *positions, const int32_t *cu,
                                const int32_t *ctx_lens, int32_t num_segs, int32_t num_rows, void *q_out, void *k_out, void *stream)
{
    const char *fn = "tetri_qk_norm_rope";
    if (!h) return tetri_fail(nullptr, TETRI_ERR_INVALID_ARG, "%s: null handle", fn);
    const void *ptrs[] = {q, k, q_out, k_out};
    const char *names[] = {"q", "k", "q_out", "k_out"};
    for (int i = 0; i < 4; ++i) {
        if (!ptrs[i]) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: %s is null", fn, names[i]);
        if (!aligned16(ptrs[i])) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: %s is not 16-byte aligned", fn, names[i]);
    }
    if (!aligned16(q_weight) || !aligned16(k_weight)) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: q_weight or k_weight is not 16-byte aligned", fn);
    const tetri_config &cfg = h->cfg;
    const int64_t q_row = (int64_t)cfg.num_q_heads * cfg.head_dim, k_row = (int64_t)cfg.num_kv_heads * cfg.head_dim;
    if (q_stride < q_row || k_stride < k_row || q_stride % 8 != 0 || k_stride % 8 != 0 || q_stride > (1ll << 40) || k_stride > (1ll << 40))
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: q_stride=%lld and k_stride=%lld have to be multiples of 8, at least %lld and %lld", fn,
                    (long long)q_stride, (long long)k_stride, (long long)q_row, (long long)k_row);
    if ((q_out == q && q_stride != q_row) || (k_out == k && k_stride != k_row))
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: in place only where the rows follow each other", fn);
    if (!(std::isfinite(eps) && eps >= 0.f)) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: eps is negative or not finite", fn);
    if (!rope) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: rope is null", fn);
    if (rope->num_pairs < 8 || rope->num_pairs > cfg.head_dim / 2 || rope->num_pairs % 8 != 0)
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: num_pairs=%d is no multiple of 8 in 8..%d", fn, rope->num_pairs, cfg.head_dim / 2);
    if (rope->num_axes < 1 || rope->num_axes > 8) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: num_axes=%d outside 1..8", fn, rope->num_axes);
    if (rope->adjacent != 0 && rope->adjacent != 1) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: adjacent must be 0 or 1", fn);
    if (num_rows < 1) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: num_rows=%d is not positive", fn, num_rows);
    if (positions ? (cu || ctx_lens) : !(cu && ctx_lens))
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: either positions or cu_chunk_q_lens and ctx_lens", fn);
    if (cu && (num_segs < 1 || num_segs > cfg.max_segs_per_chunk))
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: num_segs=%d outside 1..%d", fn, num_segs, cfg.max_segs_per_chunk);
    RopeParams p;
    for (int i = 0; i < TETRI_ROPE_PAIRS; ++i) {
        const bool used = i < rope->num_pairs;
        p.freq[i] = used ? rope->freq[i] : 0.f;
        p.axis[i] = used ? rope->axis[i] : 0;
        if (!std::isfinite(p.freq[i])) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: freq[%d] is not finite", fn, i);
        if (p.axis[i] >= rope->num_axes) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: axis[%d]=%d of %d axes", fn, i, p.axis[i], rope->num_axes);
    }
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != h->device)
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: the handle was created on device %d, the current device is %d", fn, h->device, dev);
    p.q = static_cast<const uint16_t *>(q); p.k = static_cast<const uint16_t *>(k);
    p.q_weight = static_cast<const uint16_t *>(q_weight); p.k_weight = static_cast<const uint16_t *>(k_weight);
    p.q_out = static_cast<uint16_t *>(q_out); p.k_out = static_cast<uint16_t *>(k_out);
    p.pos = positions; p.cu = cu; p.ctx = ctx_lens;
    p.q_stride = q_stride; p.k_stride = k_stride;
    p.eps = eps;
    p.S = num_segs; p.rows = num_rows; p.Hq = cfg.num_q_heads; p.Hkv = cfg.num_kv_heads;
    p.pairs = rope->num_pairs; p.adjacent = rope->adjacent;
    // A row's heads go to one wavefront where rows are many (its cosines and sines are worked out once), otherwise to as many as fill eight places of
    // a compute unit, down to the heads of one instruction each.
    const int64_t per_inst = 512 / cfg.head_dim, insts = (p.Hq + p.Hkv + per_inst - 1) / per_inst;
    const int64_t want = std::max<int64_t>(1, std::min(insts, 8 * (int64_t)std::max(h->num_cus, 1) / num_rows));
    p.per_split = (int32_t)((insts + want - 1) / want);
    p.splits = (int32_t)((insts + p.per_split - 1) / p.per_split);
    p.splits_magic = p.splits <= 1 ? 0u : (uint32_t)((0x100000000ull + p.splits - 1) / p.splits);
    // More than 64 MB of rows: read past the caches, where what is written then finds room, and what is read next.  (8192 rows of 32/8 heads 38.6 -> 32.7 us, with
    // the chunk's attention behind it 116.9 -> 115.0; but 512 rows of 40 heads 7.3 and 7.9, with attention 31.1 and 32.0.  Writing past the caches is faster alone, 32.1
    // and 6.4, and slower with the attention that reads it: 121.3.)
    p.past_caches = (q_row + k_row) * 2 * num_rows > (64ll << 20);
    if ((uint64_t)num_rows * p.splits * p.splits + 4ull * p.splits >= 0x7fffffffull)
        return tetri_fail(h, TETRI_ERR_INVALID_ARG, "%s: too many rows for one launch", fn);
    hipError_t e = tetri_launch_rope(cfg.head_dim, p, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return tetri_fail(h, TETRI_ERR_HIP, "%s: launch failed: %s", fn, hipGetErrorString(e));
    return TETRI_OK;
}

}  // extern "C"
