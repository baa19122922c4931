// Attention over a cache held in 8 bits: row i of a sequence's block sees the cached tokens and rows 0 .. i of the block.
#pragma once

#include "kv_quant.h"
#include "misc_kernels.h"

namespace hsd {

struct QuantAttn {
  QuantKV kv;
  int n_seq, total_q, n_slots, max_blocks, n_q_heads;
  const int32_t *cu_q, *seq_slot, *seq_len, *block_table;
  int64_t q_stride, o_stride;
  float scale;   // log2(e) times the softmax scale
};

// grid: (total_q, ceil(n_q_heads / 4)), block 256: a wave per row and query head, a lane per key and per dimension
template <typename T>
__global__ void __launch_bounds__(256) k_attn_quant(QuantAttn a, const T *__restrict__ q, T *__restrict__ o) {
  const int lane = threadIdx.x & 63, head = blockIdx.y * 4 + (threadIdx.x >> 6), r = blockIdx.x;
  if (head >= a.n_q_heads) return;
  const int h = head / (a.n_q_heads / a.kv.n_kv_heads), s = seq_of_row(a.cu_q, a.n_seq, r), sl = slot_of(a.seq_slot, s, a.n_slots);
  const int n_keys = min(a.seq_len[sl] + (r - a.cu_q[s]) + 1, a.max_blocks * kBlk);
  const T *qr = q + r * a.q_stride + head * kHd;
  float m = -INFINITY, l = 0.f, acc = 0.f;
  for (int j0 = 0; j0 < n_keys; j0 += kWave) {
    const int j = j0 + lane;
    int id = j < n_keys ? a.block_table[static_cast<size_t>(sl) * a.max_blocks + j / kBlk] : -1;
    if (id >= a.kv.n_blocks) id = -1;
    float score = -INFINITY;
    if (id >= 0) {
      const int page = id * a.kv.n_kv_heads + h;
      const uint8_t *kp = a.kv.k_codes + static_cast<size_t>(page) * kPageCodes + j % kBlk * 16;
      float dot = 0.f;
      for (int d = 0; d < kHd; d += 4) {
        float x[4], y[4];
        dequant4(*reinterpret_cast<const uint32_t *>(kp + d / 16 * 256 + d % 16), 1.f, x);
        quant_load4(qr + d, y);
        for (int e = 0; e < 4; ++e) dot = fmaf(x[e], y[e], dot);
      }
      score = dot * a.kv.k_scale[page] * a.scale;
    }
    const float m_new = fmaxf(m, wave_max(score));
    if (!__any(id >= 0)) continue;
    const float p = id >= 0 ? exp2f(score - m_new) : 0.f, corr = m == -INFINITY ? 0.f : exp2f(m - m_new);
    l = l * corr + wave_sum(p);
    acc *= corr;
    for (int i = 0; i < kWave; ++i) {
      const int b = __builtin_amdgcn_readlane(id, i);
      if (b < 0) continue;
      const int page = b * a.kv.n_kv_heads + h, tok = i % kBlk;
      const float x = __builtin_amdgcn_cvt_f32_fp8(a.kv.v_codes[static_cast<size_t>(page) * kPageCodes + (tok >> 2) * 256 + (lane >> 2) * 16 + (lane & 3) * 4 + (tok & 3)], 0);
      acc = fmaf(__shfl(p, i, kWave) * a.kv.v_scale[page], x, acc);
    }
    m = m_new;
  }
  o[r * a.o_stride + head * kHd + lane] = from_f32<T>(l == 0.f ? 0.f : acc / l);
}

}  // namespace hsd
