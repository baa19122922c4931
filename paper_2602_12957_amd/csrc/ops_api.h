// C entries of the operators that run without a decoder context: rows placed in pages, the 8-bit cache, token scores.
#pragma once

#include "ops_launch.h"

extern "C" {

int hsd_kv_reserve(void *stream, const hsd_kv_pool *pool, const hsd_batch *b, int32_t *row_slot, int32_t *row_pos) {
  int rc = check_rows(b);
  if (rc == HSD_OK) rc = check_free_list(pool);
  if (rc != HSD_OK) return rc;
  if (b->status == nullptr || (row_slot == nullptr && b->total_q > 0)) return HSD_EINVAL;
  const KvPlace p{b->n_seq, b->total_q, b->n_slots, b->max_blocks_per_seq, pool->n_blocks, b->cu_q, b->seq_slot, b->seq_len,
                  b->block_table, pool->free_list, pool->free_count, b->status, row_slot, row_pos};
  hipLaunchKernelGGL(k_kv_place, dim3(1), dim3(1024), 0, static_cast<hipStream_t>(stream), p);
  HSD_LAUNCH_CHECK();
  if (b->total_q > kPlaceRows) {
    hipLaunchKernelGGL(k_kv_place_rows, dim3((b->total_q + 1023) / 1024), dim3(256), 0, static_cast<hipStream_t>(stream), p);
    HSD_LAUNCH_CHECK();
  }
  return HSD_OK;
}

int hsd_kv_commit_rows(void *stream, const hsd_kv_pool *pool, const hsd_batch *b) {
  int rc = check_rows(b);
  if (rc == HSD_OK) rc = check_free_list(pool);
  if (rc != HSD_OK) return rc;
  hipLaunchKernelGGL(k_kv_commit, dim3(1), dim3(1024), 0, static_cast<hipStream_t>(stream), b->n_seq, b->cu_q, b->seq_slot, b->n_slots,
                     b->seq_len, b->block_table, b->max_blocks_per_seq, pool->n_blocks, pool->free_list, pool->free_count,
                     b->accept_len, static_cast<const int32_t *>(nullptr), static_cast<int32_t *>(nullptr), b->accept_len == nullptr ? 1 : 0);
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

int hsd_kv_quant_append(void *stream, const hsd_kv_quant *kv, int32_t n_rows, const int32_t *row_slot, int32_t dtype, const void *k, const void *v,
                        int64_t k_stride, int64_t v_stride, int32_t *status) {
  const int rc = check_quant(kv);
  if (rc != HSD_OK) return rc;
  if (n_rows < 0 || !is_type(dtype)) return HSD_EINVAL;
  if (n_rows > kMostPlacedRows) return HSD_ERANGE;
  if (n_rows == 0) return HSD_OK;
  const int64_t width = static_cast<int64_t>(kv->n_kv_heads) * HSD_HEAD_DIM;
  if (row_slot == nullptr || k == nullptr || v == nullptr || k_stride < width || v_stride < width) return HSD_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == HSD_BF16)
    return launch_append(st, quant_pages(kv), n_rows, row_slot, QuantRows<bf16>{static_cast<const bf16 *>(k), static_cast<const bf16 *>(v), k_stride, v_stride}, status);
  return launch_append(st, quant_pages(kv), n_rows, row_slot, QuantRows<float>{static_cast<const float *>(k), static_cast<const float *>(v), k_stride, v_stride}, status);
}

int hsd_kv_quant_read(void *stream, const hsd_kv_quant *kv, int32_t n_rows, const int32_t *row_slot, int32_t dtype, void *k, void *v,
                      int64_t k_stride, int64_t v_stride) {
  const int rc = check_quant(kv);
  if (rc != HSD_OK) return rc;
  if (n_rows < 0 || !is_type(dtype)) return HSD_EINVAL;
  if (n_rows > kMostPlacedRows) return HSD_ERANGE;
  if (n_rows == 0) return HSD_OK;
  const int64_t width = static_cast<int64_t>(kv->n_kv_heads) * HSD_HEAD_DIM;
  if (row_slot == nullptr || k == nullptr || v == nullptr || k_stride < width || v_stride < width) return HSD_EINVAL;
  const int span = run_span(n_rows, kv->n_kv_heads);
  const dim3 grid((static_cast<unsigned>(n_rows) + 4 * span - 1) / (4 * span), kv->n_kv_heads);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == HSD_BF16)
    hipLaunchKernelGGL((k_quant_read<bf16>), grid, dim3(256), 0, st, quant_pages(kv), n_rows, span, row_slot, static_cast<bf16 *>(k),
                       static_cast<bf16 *>(v), k_stride, v_stride);
  else
    hipLaunchKernelGGL((k_quant_read<float>), grid, dim3(256), 0, st, quant_pages(kv), n_rows, span, row_slot, static_cast<float *>(k),
                       static_cast<float *>(v), k_stride, v_stride);
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

size_t hsd_kv_quant_attention_bytes(const hsd_kv_quant *kv, const hsd_batch *b, int32_t n_q_heads) {
  if (check_quant(kv) != HSD_OK || check_rows(b) != HSD_OK || check_heads(kv, b, n_q_heads) != HSD_OK) return 0;
  const QuantPlan bf = plan_quant_attention(kv, b, n_q_heads, false), f32 = plan_quant_attention(kv, b, n_q_heads, true);
  return std::max(bf.part_rows, f32.part_rows) * kPartRowBytes;
}

int hsd_kv_quant_attention(void *stream, const hsd_kv_quant *kv, const hsd_batch *b, int32_t n_q_heads, int32_t dtype, float softmax_scale,
                           const void *q, int64_t q_stride, void *out, int64_t out_stride, void *ws, size_t ws_bytes) {
  int rc = check_quant(kv);
  if (rc == HSD_OK) rc = check_rows(b);
  if (rc != HSD_OK) return rc;
  if (!is_type(dtype) || !std::isfinite(softmax_scale * kLog2e)) return HSD_EINVAL;
  if ((rc = check_heads(kv, b, n_q_heads)) != HSD_OK) return rc;
  if (b->total_q == 0) return HSD_OK;
  const int64_t width = static_cast<int64_t>(n_q_heads) * HSD_HEAD_DIM;
  if (q == nullptr || out == nullptr || q_stride < width || out_stride < width) return HSD_EINVAL;
  const QuantPlan p = plan_quant_attention(kv, b, n_q_heads, dtype == HSD_FP32);
  if ((rc = check_workspace(ws, ws_bytes, p.part_rows * kPartRowBytes)) != HSD_OK) return rc;
  return run_quant_attention(static_cast<hipStream_t>(stream), kv, b, n_q_heads, dtype, softmax_scale * kLog2e, q, q_stride, out, out_stride, ws, p);
}

size_t hsd_token_logprobs_bytes(int32_t n_rows, int32_t vocab, int32_t n_top) {
  if (n_rows < 0 || vocab < 1 || n_top < 0 || n_top > HSD_MAX_TOP) return 0;
  const int parts = plan_scores(n_rows, vocab, 4).n_parts;
  return parts > 1 ? static_cast<size_t>(n_rows) * parts * (sizeof(float4) + n_top * sizeof(uint64_t)) : 0;
}

int hsd_token_logprobs(void *stream, int32_t n_rows, int32_t vocab, int32_t dtype, const void *logits, int64_t row_stride, const int32_t *tokens,
                       float *logprob, float *entropy, int32_t n_top, int32_t *top_ids, float *top_logprobs, void *ws, size_t ws_bytes) {
  if (n_rows < 0 || vocab < 1 || n_top < 0 || !is_type(dtype) || row_stride < vocab) return HSD_EINVAL;
  if (n_top > HSD_MAX_TOP || vocab > (1 << 30) || n_rows > kMostScoredRows) return HSD_ERANGE;
  if (n_rows == 0) return HSD_OK;
  if (logits == nullptr || tokens == nullptr || logprob == nullptr || entropy == nullptr) return HSD_EINVAL;
  if (n_top > 0 && (top_ids == nullptr || top_logprobs == nullptr)) return HSD_EINVAL;
  const int rc = check_workspace(ws, ws_bytes, hsd_token_logprobs_bytes(n_rows, vocab, n_top));
  if (rc != HSD_OK) return rc;
  const ScorePlan p = plan_scores(n_rows, vocab, dtype == HSD_BF16 ? 8 : 4);
  float4 *sums = static_cast<float4 *>(ws);
  const TokenScores a{n_rows, vocab, n_top, p.n_parts, p.part_len, row_stride, tokens, logprob, entropy, top_logprobs, top_ids, sums,
                      reinterpret_cast<uint64_t *>(sums + static_cast<size_t>(n_rows) * p.n_parts)};
  hipStream_t st = static_cast<hipStream_t>(stream);
  return dtype == HSD_BF16 ? launch_scores(st, a, p, static_cast<const bf16 *>(logits)) : launch_scores(st, a, p, static_cast<const float *>(logits));
}

size_t hsd_workspace_quant_bytes(const hsd_model_desc *desc, int32_t max_total_q, int32_t max_n_seq, int32_t max_blocks_per_seq) {
  if (hsd_validate_model(desc) != HSD_OK || max_total_q < 1 || max_n_seq < 1 || max_blocks_per_seq < 1) return 0;
  return carve_quant(*desc, max_total_q, max_n_seq, max_blocks_per_seq, nullptr).total;
}

int hsd_verify_quant(hsd_ctx *ctx, void *stream, const hsd_kv_pool *pool, const hsd_kv_quant *layers, const hsd_batch *batch, void *ws,
                     size_t ws_bytes) {
  return quant_pass(ctx, stream, pool, layers, batch, ws, ws_bytes, /*prefill=*/false);
}

int hsd_prefill_quant(hsd_ctx *ctx, void *stream, const hsd_kv_pool *pool, const hsd_kv_quant *layers, const hsd_batch *batch, void *ws,
                      size_t ws_bytes) {
  return quant_pass(ctx, stream, pool, layers, batch, ws, ws_bytes, /*prefill=*/true);
}

}  // extern "C"
