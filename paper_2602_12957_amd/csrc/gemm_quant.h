// Products of rows and weights that are held in 8 bits.
//
// out[m][n] = sum over blocks b of 128 columns of 2^(sa[m][b] - 127) * sw[n / 128][b] * sum_k a[m][k] w[n][k]
#pragma once

#include "rows_quant.h"

namespace hsd {

struct WeightQuant {
  const uint8_t *codes;
  const void *scale;        // bytes (powers of two) or floats
  int64_t code_stride, scale_stride;
  int32_t bytes;            // whether they are bytes
};
// A block's sum times its row's and its weights' scales (exponents together: each alone may leave fp32's range)
__device__ __forceinline__ float scaled(float sum, uint32_t row_byte, const WeightQuant &w, int64_t i) {
  if (w.bytes) return ldexpf(sum, static_cast<int>(row_byte) + static_cast<const uint8_t *>(w.scale)[i] - 254);
  return ldexpf(sum * static_cast<const float *>(w.scale)[i], static_cast<int>(row_byte) - 127);
}

__device__ __forceinline__ float dot4(uint32_t a, uint32_t b, float s) {
  float x[4], y[4];
  dequant4(a, 1.f, x), dequant4(b, 1.f, y);
#pragma unroll
  for (int i = 0; i < 4; ++i) s = __builtin_fmaf(x[i], y[i], s);
  return s;
}

// One output of a row and a weight row
__device__ __forceinline__ float plain_product(const RowsQuant &a, const WeightQuant &w, int64_t m, int64_t n, int blocks) {
  float sum = 0.f;
  for (int b = 0; b < blocks; ++b) {
    const uint32_t *x = reinterpret_cast<const uint32_t *>(a.codes + m * a.code_stride + b * kQuantBlock);
    const uint32_t *y = reinterpret_cast<const uint32_t *>(w.codes + n * w.code_stride + b * kQuantBlock);
    float s = 0.f;
    for (int i = 0; i < kQuantBlock / 4; ++i) s = dot4(x[i], y[i], s);
    sum += scaled(s, a.scale[m * a.scale_stride + b], w, n / kQuantBlock * w.scale_stride + b);
  }
  return sum;
}

// A thread an output: grid (columns / 256, rows)
template <typename T>
__global__ void __launch_bounds__(256) k_quant_linear(const RowsQuant a, const WeightQuant w, int64_t m0, int n_out, int blocks, T *out, int64_t out_stride) {
  const int64_t m = m0 + blockIdx.y;
  const int n = blockIdx.x * 256 + threadIdx.x;
  if (n < n_out) out[m * out_stride + n] = from_f32<T>(plain_product(a, w, m, n, blocks));
}

// silu(gate) * up of 128 columns of one row, to 8 bits: grid (columns / 128, rows)
__global__ void __launch_bounds__(128) k_quant_gated(const RowsQuant a, const WeightQuant w, int64_t m0, int d_ffn, int blocks, const RowsQuant out) {
  __shared__ float y[kQuantBlock];
  const int64_t m = m0 + blockIdx.y;
  const int t = threadIdx.x, n = blockIdx.x * kQuantBlock + t;
  const float g = plain_product(a, w, m, n, blocks), u = plain_product(a, w, m, d_ffn + n, blocks);
  y[t] = g / (1.f + expf(-g)) * u;
  __syncthreads();
  if (t < 16) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = y[8 * t + i];
    store_codes8(out, m, blockIdx.x * kQuantBlock + 8 * t, v);
  }
}

}  // namespace hsd
