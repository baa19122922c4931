// What the operators around the 8-bit cache and the token scores check, how their work is split, and their launches.
#pragma once

namespace {

// A launch has fewer than 2^32 threads: rows that take 4 and 256 of them each.  Positions (cached tokens and rows) stay below 2^31.
constexpr int kMostPlacedRows = 1 << 29, kMostScoredRows = (1 << 24) - 1;
constexpr int kMostTableBlocks = (INT32_MAX - kMostPlacedRows) / HSD_KV_BLOCK_TOKENS;

int check_rows(const hsd_batch *b) {
  if (b == nullptr || b->n_seq < 1 || b->total_q < 0 || b->max_blocks_per_seq < 1 || b->n_slots < 1) return HSD_EINVAL;
  if (b->seq_slot == nullptr && b->n_slots < b->n_seq) return HSD_EINVAL;
  if (b->n_seq > HSD_MAX_SEQ || b->total_q > kMostPlacedRows || b->max_blocks_per_seq > kMostTableBlocks) return HSD_ERANGE;
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
  return n_q_heads > 1024 || static_cast<int64_t>(b->total_q) * n_q_heads > INT32_MAX / 4 ? HSD_ERANGE : HSD_OK;
}

constexpr int kSplitBlocks = 256;   // keys are split over workgroups where tables hold more

// How an attention call is split.  Lengths are on the device: the plan goes by rows, heads and what the tables can hold.
struct QuantPlan {
  int ct, waves, n_tiles, n_splits;
  int parts;          // of a bf16 call's probabilities
  size_t part_rows;   // rows of the workspace's parts
};
QuantPlan plan_quant_attention(const hsd_kv_quant *kv, const hsd_batch *b, int32_t n_q_heads, bool f32) {
  const int64_t group = n_q_heads / kv->n_kv_heads, cols = b->total_q * group;
  QuantPlan p;
  // tiles that have columns, about (each sequence may have an empty one more)
  auto real_tiles = [&](int64_t c) { return (cols <= c * b->n_seq ? b->n_seq : cols / c + b->n_seq / 2) * kv->n_kv_heads; };
  // 64 columns a wave where that still gives every SIMD its two waves: they share what making operands of pages costs.  Below,
  // 32, of which a unit holds 16 waves.  us a call, 64 / 32 columns, by tiles of 64 (16 heads on 4): 576 (16 blocks of up to 257 rows
  // on 1055 keys) 38.8 / 30.3, 1024 (4 of 2000 rows) 82.0 / 72.8, 2112 (64 of up to 256 rows on 1280) 96.2 / 104.7.
  const int64_t tiles64 = real_tiles(64);
  p.ct = f32 || tiles64 < 2048 ? 1 : 2;
  p.n_tiles = static_cast<int>(cols / (32 * p.ct) + b->n_seq);
  const int64_t groups = p.n_tiles * static_cast<int64_t>(kv->n_kv_heads), max_pairs = (b->max_blocks_per_seq + 1) / 2;
  const int64_t real = p.ct == 2 ? tiles64 : real_tiles(32);
  // keys over the workgroups where a wave of a full workgroup would take more than eight steps and the chip is not full
  p.n_splits = 1;
  if (b->max_blocks_per_seq > kSplitBlocks && real < 512) p.n_splits = static_cast<int>(std::min<int64_t>({(511 + real) / real, (max_pairs + 63) / 64, kMaxSplits}));
  // keys over the waves: as many as let all workgroups run at once (but for a 64th of them, which start as the first ones end), and
  // two at least (late tiles of a block see more keys than early ones).  us a call, 16 heads on 4: 810 tiles (4 blocks of 401 rows on 1055
  // keys) 24.2 / 23.1 / 23.5 / 33.4 with 2 / 3 / 4 / 5 waves, of which 5 leave room for 768; 1026 (one of 2049 on 4127) 77.5 / 73.5 with 3 / 4; 1228 (16 of up to 257
  // on 1055) 29.2 / 27.7 / 28.0 / 36.8 with 2 / 3 / 4 / 5; 4008 (4 of 2000) 89 / 70 / 72 with 1 / 2 / 3.
  const int most = quant_attn_waves(f32, p.ct);
  const int64_t all = real * p.n_splits, a_unit = (all - all / 64 + 255) / 256;
  p.waves = static_cast<int>(std::max<int64_t>(std::min<int64_t>({most, std::max<int64_t>(most / a_unit, 2), max_pairs}), 1));
  // two parts where the keys are split and a sequence's columns are one tile, so that pages are read once and wait for memory: 107.9 us
  // where one part takes 105.3 (8 rows on 131072 keys); with two tiles and 16 a sequence 37.7 / 30.9 (8 of 16 rows on 8192) and 44.8 / 35.7
  p.parts = p.n_splits > 1 && cols <= 32 * static_cast<int64_t>(b->n_seq) ? 2 : 1;
  p.part_rows = p.n_splits > 1 ? static_cast<size_t>(groups) * p.n_splits * 32 * p.ct : 0;
  return p;
}

template <typename T, int CT, int NP>
int launch_quant_attention(hipStream_t st, const QuantAttn &a, const QuantPlan &p, const T *q, T *out) {
  auto kern = k_attn_quant<T, CT, NP>;
  const int lds = quant_attn_lds(p.waves);
  static const hipError_t attr_rc = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                        quant_attn_lds(quant_attn_waves(std::is_same<T, float>::value, CT)));
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
  // (16 rows of 32768 in fp32: 8.2 us in one part, 7.1 and 3.9 to join them in two)
  p.n_parts = static_cast<int>(std::max<int64_t>(std::min<int64_t>({kScoreParts, 512 / std::max<int64_t>(n_rows, 1), vocab / 32768}), 1));
  p.part_len = static_cast<int>(vocab);
  if (p.n_parts > 1) {
    const int64_t unit = 64 * piece;   // (no part is empty: 64 * 8 * 16 is less than a part)
    p.part_len = static_cast<int>((vocab + p.n_parts * unit - 1) / (p.n_parts * unit) * unit);
    p.n_parts = static_cast<int>((vocab + p.part_len - 1) / p.part_len);
  }
  // us a call by waves a workgroup, 16 / 8 / 4: one fp32 row of 200000 20.5 / 21.4 / 24.8, 700 bf16 rows of 32768 27.2 / 19.5 / 20.3, 1856
  // 70.3 / 52.8 / 41.5 (all in turn among other sizes, caches cold)
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

constexpr float kLog2e = 1.4426950408889634f;
constexpr size_t kPartRowBytes = (HSD_HEAD_DIM + 2) * sizeof(float);
// What any plan's parts take at most: keys are split where there are fewer than 512 tiles with columns, into 511 + 511 runs with
// theirs at most, at most twice as many with the tiles that have none, of 32 columns
constexpr size_t kMostPartRows = size_t{2} * 1022 * 32;

// Attention of one layer; exponents of 2 are scale2 times the products
int run_quant_attention(hipStream_t st, const hsd_kv_quant *kv, const hsd_batch *b, int32_t n_q_heads, int32_t dtype, float scale2, const void *q,
                        int64_t q_stride, void *out, int64_t out_stride, void *ws, const QuantPlan &p) {
  float *part = static_cast<float *>(ws);
  const QuantAttn a{quant_pages(kv), b->n_seq, b->total_q, b->n_slots, b->max_blocks_per_seq, n_q_heads, n_q_heads / kv->n_kv_heads, b->cu_q,
                    b->seq_slot, b->seq_len, b->block_table, q_stride, out_stride, std::max(std::fabs(scale2), 1.2e-38f),
                    std::signbit(scale2) ? 0x80000000u : 0u, p.n_tiles, p.n_splits, heads_log(kv->n_kv_heads), group_mul(n_q_heads / kv->n_kv_heads),
                    waves_mul(p.waves), part, reinterpret_cast<float2 *>(part + p.part_rows * HSD_HEAD_DIM)};
  if (dtype == HSD_BF16) {
    const bf16 *x = static_cast<const bf16 *>(q);
    bf16 *y = static_cast<bf16 *>(out);
    if (p.parts == 2) return launch_quant_attention<bf16, 1, 2>(st, a, p, x, y);
    return p.ct == 1 ? launch_quant_attention<bf16, 1, 1>(st, a, p, x, y) : launch_quant_attention<bf16, 2, 1>(st, a, p, x, y);
  }
  return launch_quant_attention<float, 1, 3>(st, a, p, static_cast<const float *>(q), static_cast<float *>(out));
}

template <typename Src>
int launch_append(hipStream_t st, const QuantKV &kv, int n_rows, const int32_t *row_slot, const Src &src, int32_t *status) {
  const int span = run_span(n_rows, kv.n_kv_heads);
  const dim3 grid((static_cast<unsigned>(n_rows) + 4 * span - 1) / (4 * span), kv.n_kv_heads);
  hipLaunchKernelGGL((k_quant_append<Src>), grid, dim3(256), 0, st, kv, n_rows, span, row_slot, src, status);
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

// What a pass on an 8-bit cache needs behind its workspace: the rows' keys and values in the model's type, their numbers, and the
// attention's parts
struct QuantWorkspace {
  void *k, *v;
  int32_t *row;
  void *parts;
  size_t total;   // with the pass's own
};
QuantWorkspace carve_quant(const hsd_model_desc &d, int64_t T, int64_t n_seq, int64_t max_blocks, void *base) {
  const size_t es = d.dtype == HSD_BF16 ? 2 : 4, pages = static_cast<size_t>((T + kBlk - 1) / kBlk) * d.n_kv_heads * kPageCodes;
  size_t off = carve(d, T, n_seq, nullptr).total;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += align_up(bytes);
    return base ? static_cast<void *>(static_cast<char *>(base) + o) : nullptr;
  };
  QuantWorkspace w;
  w.k = take(pages * es), w.v = take(pages * es);
  w.row = static_cast<int32_t *>(take(T * sizeof(int32_t)));
  w.parts = take(max_blocks > kSplitBlocks ? kMostPartRows * kPartRowBytes : 0);
  w.total = off;
  return w;
}

}  // namespace
