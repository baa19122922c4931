// Scores of given tokens under rows of logits: log probability, entropy of the row, its most probable tokens.
#pragma once

#include "common.h"

namespace hsd {

struct TokenScores {
  int n_rows, vocab, n_top;
  int64_t stride;
  const int32_t *tokens;
  float *logprob, *entropy, *top_logprob;
  int32_t *top_id;
};

// (value, index) order of the alternatives: larger value first, lower index among equals
__device__ __forceinline__ bool score_before(float va, int ia, float vb, int ib) { return va > vb || (va == vb && ia < ib); }

// One workgroup a row.  m = max x, Z = sum e^(x - m), W = sum (x - m) e^(x - m): log p = x - m - ln Z, entropy = ln Z - W / Z.
// grid: n_rows, block 256
template <typename T>
__global__ void __launch_bounds__(256) k_token_scores(TokenScores a, const T *__restrict__ logits) {
  __shared__ float s_v[4], s_w[4];
  __shared__ int s_i[4];
  const int r = blockIdx.x, t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const T *x = logits + r * a.stride;
  float m = -INFINITY;
  for (int i = t; i < a.vocab; i += 256) m = fmaxf(m, to_f32(x[i]));
  m = wave_max(m);
  if (lane == 0) s_v[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(s_v[0], s_v[1]), fmaxf(s_v[2], s_v[3]));
  __syncthreads();
  float z = 0.f, w = 0.f;
  for (int i = t; i < a.vocab; i += 256) {
    const float v = to_f32(x[i]);
    if (v == -INFINITY) continue;
    const float d = v - m, e = expf(d);
    z += e;
    if (!(e <= 0.f)) w = fmaf(d, e, w);
  }
  z = wave_sum(z), w = wave_sum(w);
  if (lane == 0) s_v[wave] = z, s_w[wave] = w;
  __syncthreads();
  z = s_v[0] + s_v[1] + s_v[2] + s_v[3], w = s_w[0] + s_w[1] + s_w[2] + s_w[3];
  const float lz = logf(z);
  __syncthreads();
  if (t == 0) {
    const int tok = a.tokens[r];
    const bool inside = tok >= 0 && tok < a.vocab;
    const float v = inside ? to_f32(x[tok]) : -INFINITY;
    a.logprob[r] = inside && z != z ? z : (v == -INFINITY ? v : v - m - lz);
    a.entropy[r] = m == -INFINITY && z == 0.f ? 0.f : lz - w / z;
  }
  float pv = INFINITY;
  int pi = -1;
  for (int j = 0; j < a.n_top; ++j) {
    float bv = -INFINITY;
    int bi = 0x7fffffff;
    for (int i = t; i < a.vocab; i += 256) {
      const float v = to_f32(x[i]);
      if (score_before(pv, pi, v, i) && score_before(v, i, bv, bi)) bv = v, bi = i;
    }
    for (int o = 32; o > 0; o >>= 1) {
      const float ov = __shfl_xor(bv, o, kWave);
      const int oi = __shfl_xor(bi, o, kWave);
      if (score_before(ov, oi, bv, bi)) bv = ov, bi = oi;
    }
    if (lane == 0) s_v[wave] = bv, s_i[wave] = bi;
    __syncthreads();
    for (int u = 0; u < 4; ++u)
      if (score_before(s_v[u], s_i[u], bv, bi)) bv = s_v[u], bi = s_i[u];
    __syncthreads();
    const bool none = bv == -INFINITY;
    if (t == 0) {
      a.top_id[static_cast<size_t>(r) * a.n_top + j] = none ? -1 : bi;
      a.top_logprob[static_cast<size_t>(r) * a.n_top + j] = none ? -INFINITY : bv - m - lz;
    }
    pv = bv, pi = none ? 0x7fffffff : bi;
  }
}

}  // namespace hsd
