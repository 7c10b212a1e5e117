// Entry points of the KV cache in 4-bit codes.  What they check and how they are launched they share with the caches of 16 and 8
// bits; the kernels they hand in.
#include "tetri_internal.h"

namespace {

constexpr Fp4Launchers kLaunchers = {tetri_launch_kv_export_fp4, tetri_launch_kv_import_fp4, tetri_launch_decode_fp4, tetri_launch_attn_fp4,
                                     tetri_launch_prefill_fp4};

}  // namespace

extern "C" {

tetri_status tetri_kv_export_fp4(tetri_ctx *h, const void *kv_pages, const int32_t *block_table, const int32_t *cu_tokens,
                                 const int32_t *first_tokens, int32_t num_reqs, int64_t total_tokens, void *buf, void *stream)
{
    return tetri_transfer_fp4_call("tetri_kv_export_fp4", h, const_cast<void *>(kv_pages), buf, block_table, cu_tokens, first_tokens, num_reqs,
                                   total_tokens, false, stream, kLaunchers);
}

tetri_status tetri_kv_import_fp4(tetri_ctx *h, const void *buf, const int32_t *block_table, const int32_t *cu_tokens,
                                 const int32_t *first_tokens, int32_t num_reqs, int64_t total_tokens, void *kv_pages_fp4,
                                 void *stream)
{
    return tetri_transfer_fp4_call("tetri_kv_import_fp4", h, kv_pages_fp4, const_cast<void *>(buf), block_table, cu_tokens, first_tokens, num_reqs,
                                   total_tokens, true, stream, kLaunchers);
}

tetri_status tetri_decode_attn_fp4(tetri_ctx *h, const void *q, const void *k_new, const void *v_new, void *kv_pages_fp4, const int32_t *block_table,
                                   const int32_t *ctx_lens, int32_t num_reqs, int32_t max_ctx_len, float scale, int32_t append, void *out,
                                   void *stream)
{
    if (append != 0 && append != 1) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "tetri_decode_attn_fp4: append must be 0 or 1");
    return tetri_decode_fp4_call("tetri_decode_attn_fp4", h, q, k_new, v_new, kv_pages_fp4, append ? kv_pages_fp4 : nullptr, block_table, ctx_lens,
                                 num_reqs, max_ctx_len, scale, out, stream, kLaunchers);
}

tetri_status tetri_chunk_prefill_attn_fp4(tetri_ctx *h, const void *q, const void *k_new, const void *v_new, void *kv_pages_fp4,
                                          const int32_t *block_table, const int32_t *cu, const int32_t *ctx_lens, int32_t num_segs, float scale,
                                          int32_t append, void *out, void *stream)
{
    if (append != 0 && append != 1) return tetri_fail(h, TETRI_ERR_INVALID_ARG, "tetri_chunk_prefill_attn_fp4: append must be 0 or 1");
    return tetri_prefill_fp4_call("tetri_chunk_prefill_attn_fp4", h, q, k_new, v_new, kv_pages_fp4, append ? kv_pages_fp4 : nullptr, block_table, cu,
                                  ctx_lens, num_segs, scale, out, stream, kLaunchers);
}

}  // extern "C"
