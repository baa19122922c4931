// C entries of the operators that run without a decoder context: rows placed in pages, the 8-bit cache, token scores.
#pragma once

#include "attn_quant.h"
#include "kv_place.h"
#include "kv_quant.h"
#include "token_scores.h"

namespace {

int check_rows(const hsd_batch *b) {
  if (b == nullptr || b->n_seq < 1 || b->total_q < 0 || b->max_blocks_per_seq < 1 || b->n_slots < 1) return HSD_EINVAL;
  if (b->seq_slot == nullptr && b->n_slots < b->n_seq) return HSD_EINVAL;
  if (b->n_seq > HSD_MAX_SEQ || b->max_blocks_per_seq > INT32_MAX / HSD_KV_BLOCK_TOKENS) return HSD_ERANGE;
  if (b->cu_q == nullptr || b->seq_len == nullptr || b->block_table == nullptr) return HSD_EINVAL;
  return b->tree_end != nullptr ? HSD_EINVAL : HSD_OK;   // chains only
}

int check_free_list(const hsd_kv_pool *p) {
  return p == nullptr || p->free_list == nullptr || p->free_count == nullptr || p->n_blocks < 1 ? HSD_EINVAL : HSD_OK;
}

int check_quant(const hsd_kv_quant *kv) {
  if (kv == nullptr || kv->k_codes == nullptr || kv->v_codes == nullptr || kv->k_scale == nullptr || kv->v_scale == nullptr) return HSD_EINVAL;
  if (kv->n_blocks < 1 || kv->n_kv_heads < 1) return HSD_EINVAL;
  if (((reinterpret_cast<uintptr_t>(kv->k_codes) | reinterpret_cast<uintptr_t>(kv->v_codes)) & 15) != 0) return HSD_EINVAL;
  if (kv->n_kv_heads > 1024 || static_cast<int64_t>(kv->n_blocks) * kv->n_kv_heads > INT32_MAX || kv->n_blocks > INT32_MAX / HSD_KV_BLOCK_TOKENS)
    return HSD_ERANGE;
  return HSD_OK;
}

QuantKV quant_pages(const hsd_kv_quant *kv) {
  return QuantKV{static_cast<uint8_t *>(kv->k_codes), static_cast<uint8_t *>(kv->v_codes), kv->k_scale, kv->v_scale, kv->n_blocks, kv->n_kv_heads};
}

// Whether `ws` will do as a workspace of `need` bytes (aligned to 256, as the callers are told; NULL if nothing is needed)
int check_workspace(const void *ws, size_t ws_bytes, size_t need) {
  if (need == 0) return HSD_OK;
  if (ws == nullptr || (reinterpret_cast<uintptr_t>(ws) & 255) != 0) return HSD_EINVAL;
  return ws_bytes < need ? HSD_ENOSPC : HSD_OK;
}

int check_heads(const hsd_kv_quant *kv, const hsd_batch *b, int32_t n_q_heads) {
  if (n_q_heads < 1 || n_q_heads % kv->n_kv_heads != 0) return HSD_EINVAL;
  return n_q_heads > 1024 || static_cast<int64_t>(b->total_q) * n_q_heads > INT32_MAX / 2 ? HSD_ERANGE : HSD_OK;
}

// How an attention call is split.  Lengths are on the device: the plan goes by rows, heads and what the tables can hold.
struct QuantPlan {
  int ct, waves, n_tiles, n_splits;
  size_t part_rows;   // rows of the workspace's parts
};
QuantPlan plan_quant_attention(const hsd_kv_quant *kv, const hsd_batch *b, int32_t n_q_heads, bool f32) {
  const int64_t group = n_q_heads / kv->n_kv_heads, cols = b->total_q * group;
  QuantPlan p;
    // tiles that have columns, about (each sequence may have an empty one more)
  auto real_tiles = [&](int64_t c) { return (cols <= c * b->n_seq ? b->n_seq : cols / c + b->n_seq / 2) * kv->n_kv_heads; };
  // 64 columns a wave where that still gives every SIMD its two waves: they share what making operands of pages costs.  Below,
  // 32, of which a unit holds 16 waves.  us a call, 64 / 32 columns, by tiles of 64 (16 heads on 4): 576 (16 blocks of up to 257 rows
  // on 1055 keys) 34.0 / 29.7, 1024 (4 of 2000 rows) 77.7 / 71.2, 2112 (64 of up to 256 rows on 1280) 95.4 / 96.6.
  const int64_t tiles64 = real_tiles(64);
  p.ct = f32 || tiles64 < 2048 ? 1 : 2;
  p.n_tiles = static_cast<int>(cols / (32 * p.ct) + b->n_seq);
  const int64_t groups = p.n_tiles * static_cast<int64_t>(kv->n_kv_heads), max_pairs = (b->max_blocks_per_seq + 1) / 2;
  const int64_t real = p.ct == 2 ? tiles64 : real_tiles(32);
  // keys over the workgroups where a wave of a full workgroup would take more than eight steps and the chip is not full
  p.n_splits = 1;
  if (max_pairs > 128 && real < 512) p.n_splits = static_cast<int>(std::min<int64_t>({(511 + real) / real, (max_pairs + 63) / 64, kMaxSplits}));
  // keys over the waves: as many as fit the chip at once, and two at least (late tiles of a block see more keys than early ones:
  // 4 blocks of 2000 rows 89 us with one wave a tile, 71 with two)
  const int most = quant_attn_waves(f32, p.ct);
  const int64_t fit = 256 * (f32 ? 8 : most) / (real * p.n_splits);
  p.waves = static_cast<int>(std::max<int64_t>(std::min<int64_t>({most, std::max<int64_t>(fit, p.ct == 2 ? 1 : 2), max_pairs}), 1));
  p.part_rows = p.n_splits > 1 ? static_cast<size_t>(groups) * p.n_splits * 32 * p.ct : 0;
  return p;
}

template <typename T, int CT>
int launch_quant_attention(hipStream_t st, const QuantAttn &a, const QuantPlan &p, const T *q, T *out) {
  auto kern = k_attn_quant<T, CT>;
  const int lds = quant_attn_lds(p.waves, CT);
  static const hipError_t attr_rc = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                        quant_attn_lds(quant_attn_waves(std::is_same<T, float>::value, CT), CT));
  if (attr_rc != hipSuccess) return HSD_EHIP;
  const unsigned groups = static_cast<unsigned>(p.n_tiles) * a.kv.n_kv_heads;
  hipLaunchKernelGGL(kern, dim3(tile_blocks(p.n_tiles, a.kv.n_kv_heads), p.n_splits), dim3(64 * p.waves), lds, st, a, q, out);
  HSD_LAUNCH_CHECK();
  if (p.n_splits > 1) {
    hipLaunchKernelGGL((k_attn_quant_join<T>), dim3(groups, 8 * CT), dim3(256), 0, st, a, 32 * CT, out);
    HSD_LAUNCH_CHECK();
  }
  return HSD_OK;
}

// How rows of logits are dealt out: in parts where few rows would leave the chip empty, to larger workgroups the fewer there are.
struct ScorePlan {
  int n_parts, part_len, waves;
};
ScorePlan plan_scores(int64_t n_rows, int64_t vocab, int piece) {
  ScorePlan p;
  // (16 rows of 32768: 7 us in one part, 6 and 4 to join them in two)
  p.n_parts = static_cast<int>(std::max<int64_t>(std::min<int64_t>({kScoreParts, 512 / std::max<int64_t>(n_rows, 1), vocab / 32768}), 1));
  p.part_len = static_cast<int>(vocab);
  if (p.n_parts > 1) {
    const int64_t unit = 64 * piece;   // (no part is empty: 64 * 8 * 16 is less than a part)
    p.part_len = static_cast<int>((vocab + p.n_parts * unit - 1) / (p.n_parts * unit) * unit);
    p.n_parts = static_cast<int>((vocab + p.part_len - 1) / p.part_len);
  }
  // us by waves a workgroup, 16 / 8 / 4: one row of 200000 21.3 / 22.5 / 28.5, 700 rows of 32768 24.0 / 20.2 / 22.7, 1856 56.6 / 47.2 / 43.4
  p.waves = n_rows * p.n_parts <= 256 ? 16 : (n_rows <= 1024 ? 8 : 4);
  return p;
}

template <typename T>
int launch_scores(hipStream_t st, const TokenScores &a, const ScorePlan &p, const T *logits) {
  const dim3 grid(static_cast<unsigned>(a.n_rows) * p.n_parts);
  if (p.waves == 16) hipLaunchKernelGGL((k_token_scores<T, 16>), grid, dim3(1024), 0, st, a, logits);
  else if (p.waves == 8) hipLaunchKernelGGL((k_token_scores<T, 8>), grid, dim3(512), 0, st, a, logits);
  else hipLaunchKernelGGL((k_token_scores<T, 4>), grid, dim3(256), 0, st, a, logits);
  HSD_LAUNCH_CHECK();
  if (p.n_parts > 1) {
    hipLaunchKernelGGL((k_token_scores_join<T>), dim3(a.n_rows), dim3(256), 0, st, a, logits);
    HSD_LAUNCH_CHECK();
  }
  return HSD_OK;
}

bool is_type(int32_t dtype) { return dtype == HSD_BF16 || dtype == HSD_FP32; }

}  // namespace

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
  if (n_rows == 0) return HSD_OK;
  const int64_t width = static_cast<int64_t>(kv->n_kv_heads) * HSD_HEAD_DIM;
  if (row_slot == nullptr || k == nullptr || v == nullptr || k_stride < width || v_stride < width) return HSD_EINVAL;
  const int span = run_span(n_rows, kv->n_kv_heads);
  const dim3 grid((static_cast<unsigned>(n_rows) + 4 * span - 1) / (4 * span), kv->n_kv_heads);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == HSD_BF16)
    hipLaunchKernelGGL((k_quant_append<bf16>), grid, dim3(256), 0, st, quant_pages(kv), n_rows, span, row_slot, static_cast<const bf16 *>(k),
                       static_cast<const bf16 *>(v), k_stride, v_stride, status);
  else
    hipLaunchKernelGGL((k_quant_append<float>), grid, dim3(256), 0, st, quant_pages(kv), n_rows, span, row_slot, static_cast<const float *>(k),
                       static_cast<const float *>(v), k_stride, v_stride, status);
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

int hsd_kv_quant_read(void *stream, const hsd_kv_quant *kv, int32_t n_rows, const int32_t *row_slot, int32_t dtype, void *k, void *v,
                      int64_t k_stride, int64_t v_stride) {
  const int rc = check_quant(kv);
  if (rc != HSD_OK) return rc;
  if (n_rows < 0 || !is_type(dtype)) return HSD_EINVAL;
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
  return std::max(bf.part_rows, f32.part_rows) * (HSD_HEAD_DIM + 2) * sizeof(float);
}

int hsd_kv_quant_attention(void *stream, const hsd_kv_quant *kv, const hsd_batch *b, int32_t n_q_heads, int32_t dtype, float softmax_scale,
                           const void *q, int64_t q_stride, void *out, int64_t out_stride, void *ws, size_t ws_bytes) {
  int rc = check_quant(kv);
  if (rc == HSD_OK) rc = check_rows(b);
  if (rc != HSD_OK) return rc;
  if (!is_type(dtype) || !std::isfinite(softmax_scale)) return HSD_EINVAL;
  if ((rc = check_heads(kv, b, n_q_heads)) != HSD_OK) return rc;
  if (b->total_q == 0) return HSD_OK;
  const int64_t width = static_cast<int64_t>(n_q_heads) * HSD_HEAD_DIM;
  if (q == nullptr || out == nullptr || q_stride < width || out_stride < width) return HSD_EINVAL;
  const QuantPlan p = plan_quant_attention(kv, b, n_q_heads, dtype == HSD_FP32);
  if ((rc = check_workspace(ws, ws_bytes, p.part_rows * (HSD_HEAD_DIM + 2) * sizeof(float))) != HSD_OK) return rc;
  float *part = static_cast<float *>(ws);
  const QuantAttn a{quant_pages(kv), b->n_seq, b->total_q, b->n_slots, b->max_blocks_per_seq, n_q_heads, n_q_heads / kv->n_kv_heads, b->cu_q,
                    b->seq_slot, b->seq_len, b->block_table, q_stride, out_stride, std::max(std::fabs(softmax_scale) * 1.4426950408889634f, 1.2e-38f),
                    std::signbit(softmax_scale) ? 0x80000000u : 0u, p.n_tiles, p.n_splits, part, reinterpret_cast<float2 *>(part + p.part_rows * HSD_HEAD_DIM)};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == HSD_BF16) {
    const bf16 *x = static_cast<const bf16 *>(q);
    bf16 *y = static_cast<bf16 *>(out);
    return p.ct == 1 ? launch_quant_attention<bf16, 1>(st, a, p, x, y) : launch_quant_attention<bf16, 2>(st, a, p, x, y);
  }
  const float *x = static_cast<const float *>(q);
  float *y = static_cast<float *>(out);
  return launch_quant_attention<float, 1>(st, a, p, x, y);
}

size_t hsd_token_logprobs_bytes(int32_t n_rows, int32_t vocab, int32_t n_top) {
  if (n_rows < 0 || vocab < 1 || n_top < 0 || n_top > HSD_MAX_TOP) return 0;
  const int parts = plan_scores(n_rows, vocab, 4).n_parts;
  return parts > 1 ? static_cast<size_t>(n_rows) * parts * (sizeof(float4) + n_top * sizeof(uint64_t)) : 0;
}

int hsd_token_logprobs(void *stream, int32_t n_rows, int32_t vocab, int32_t dtype, const void *logits, int64_t row_stride, const int32_t *tokens,
                       float *logprob, float *entropy, int32_t n_top, int32_t *top_ids, float *top_logprobs, void *ws, size_t ws_bytes) {
  if (n_rows < 0 || vocab < 1 || n_top < 0 || !is_type(dtype) || row_stride < vocab) return HSD_EINVAL;
  if (n_top > HSD_MAX_TOP || vocab > (1 << 30)) return HSD_ERANGE;
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

}  // extern "C"
