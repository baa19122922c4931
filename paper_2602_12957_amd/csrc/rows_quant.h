// Rows and weights held in 8 bits: made, normalised, read.
//
// A row of `dim` values is held in blocks of 128: e4m3 codes, the last block padded with zeros, and one byte a block for a power of
// two: value = code * 2^(byte - 127), byte - 127 the least e in -100 .. 119 with 448 * 2^e >= the largest finite magnitude of the
// block (0 for a block of zeros), as the 8-bit cache's pages have it (scale_exp).  A power of two costs no accuracy (codes are floating point: a value's step is 2^-4 of it down to
// 2^-6 * 2^e), the matrix unit applies it by itself (its byte operands are these bytes), and a value is exact in bf16.  NaN and infinities are
// held as NaN, so that what is computed from them shows it.
#pragma once

#include "common.h"
#include "kv_quant.h"

namespace hsd {

constexpr int kQuantBlock = 128;

struct RowsQuant {
  uint8_t *codes, *scale;             // rows code_stride and scale_stride bytes apart
  int64_t code_stride, scale_stride;
};

// magnitude of y that counts for its block's scale: infinities and NaN do not
__device__ __forceinline__ float finite_mag(float y) { return fabsf(y) < INFINITY ? fabsf(y) : 0.f; }
// y * 2^-e as a code's argument: at most 448 in magnitude (larger ones, with the largest e, as that), or NaN
__device__ __forceinline__ float code_arg(float y, float inv) { return fabsf(y) < INFINITY ? __builtin_amdgcn_fmed3f(y * inv, -448.f, 448.f) : NAN; }
__device__ __forceinline__ float two_to_byte(uint32_t b) { return b ? __uint_as_float(b << 23) : 0x1p-127f; }          // 2^(b - 127)

// largest value over a row of 16 lanes, in all of them
__device__ __forceinline__ float max16(float x) {
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x128, 0xf, 0xf, true)));   // row_ror:8
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x124, 0xf, 0xf, true)));
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x122, 0xf, 0xf, true)));
  return fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x121, 0xf, 0xf, true)));
}

// x in T, nearest, ties to even; NaN stays NaN
template <typename T>
__device__ __forceinline__ T rounded(float x) {
  if constexpr (sizeof(T) == 4) return x;
  else return __builtin_bit_cast(T, static_cast<__bf16>(x));
}

// Eight values from column c of a row of dim (those behind its end as 0)
template <typename T>
__device__ __forceinline__ void load8(const T *row, int c, int dim, float *v) {
  if (c + 8 <= dim) {
    quant_load4(row + c, v), quant_load4(row + c + 4, v + 4);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < dim ? to_f32(row[c + i]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T *row, int c, int dim, const float *v) {
  if (c + 8 <= dim) {
    if constexpr (sizeof(T) == 4) {
      quant_store4(row + c, v), quant_store4(row + c + 4, v + 4);
    } else {
      typedef __bf16 b8 __attribute__((ext_vector_type(8), aligned(2)));
      const floatx8 f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
      *reinterpret_cast<b8 *>(row + c) = __builtin_convertvector(f, bf16x8);
    }
  } else {
    for (int i = 0; i < 8; ++i)
      if (c + i < dim) row[c + i] = rounded<T>(v[i]);
  }
}

// Eight values of a block that 16 neighbouring lanes hold, to codes; the first of the lanes writes the block's byte
__device__ __forceinline__ void store_codes8(const RowsQuant &out, int64_t r, int c, const float *y) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_mag(y[i]));
  top = max16(top);
  const int e = scale_exp(top);
  const float inv = exp2_int(-e);
  uint2 q;
  q.x = quant4(code_arg(y[0], inv), code_arg(y[1], inv), code_arg(y[2], inv), code_arg(y[3], inv));
  q.y = quant4(code_arg(y[4], inv), code_arg(y[5], inv), code_arg(y[6], inv), code_arg(y[7], inv));
  *reinterpret_cast<uint2 *>(out.codes + r * out.code_stride + c) = q;
  if ((c & (kQuantBlock - 1)) == 0) out.scale[r * out.scale_stride + c / kQuantBlock] = static_cast<uint8_t>(e + 127);
}

// y in 32 bits, cut towards zero with the last bit set where anything was cut: rounded once more, to fewer bits, it is y rounded once
__device__ __forceinline__ float to_odd(double y) {
  const float f = static_cast<float>(y);
  const double back = f;
  const uint32_t u = __float_as_uint(f);
  return back == y ? f : __uint_as_float((fabs(back) > fabs(y) ? u - 1 : u) | 1);
}

struct NormRows {
  int64_t n_rows;
  int32_t dim;
  int32_t norm;                        // 0: the values as they are
  const float *gain;                   // or nullptr: 1
  double eps;
  int64_t x_stride, res_stride, sum_stride;
  RowsQuant out;
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// y = h * gain / sqrt(mean(h^2) + eps), h = x + residual, to 8 bits; h to `sum`.  In 64 bits up to the values that are rounded to codes: a code of a value next to
// a border then is the definition's, squares of any row stay in range, and the memory is what such a call waits for all the same (32772 rows of
// 1024 in bf16 beside a read of the rows made: in 32 bits 69.0 us, in 64 76.7).
//
// `wpr` waves a row, its values in registers between the two looks at them: 8 R a lane (a lane has 8 neighbouring columns of each 512 wpr; 16 lanes
// a block).  R = 0: any width, read twice.  Grid: rows / (blockDim / (64 wpr)).
template <typename TX, typename TR, int R>
__global__ void __launch_bounds__(R == 4 ? 512 : 1024) k_quant_rows(const NormRows a, int wpr, const TX *x, const TR *res, TR *sum) {
  __shared__ double part[16];
  const int t = threadIdx.x, in_row = t % (64 * wpr), step = 512 * wpr;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * (blockDim.x / (64 * wpr)) + t / (64 * wpr);
  if (r >= a.n_rows) return;   // (whole waves; with more than one a row a workgroup has one row)
  const TX *xr = x + r * a.x_stride;
  const TR *rr = res ? res + r * a.res_stride : nullptr;
  TR *sr = sum ? sum + r * a.sum_stride : nullptr;
  const int width = (a.dim + kQuantBlock - 1) / kQuantBlock * kQuantBlock;
  struct Part {   // eight columns
    float x[8], res[8];
    __device__ __forceinline__ double h(int i, bool added) const { return added ? static_cast<double>(x[i]) + static_cast<double>(res[i]) : x[i]; }
  };
  auto take = [&](int c, Part &p) {
    load8(xr, c, a.dim, p.x);
    if (rr) load8(rr, c, a.dim, p.res);
  };
  Part p[R ? R : 1];
  float gain[R ? R : 1][8];
  double ss = 0., rstd = 1.;
  auto square = [&](const Part &v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double h = v.h(i, rr != nullptr);
      ss = __builtin_fma(h, h, ss);
    }
  };
  if constexpr (R > 0) {
#pragma unroll
    for (int k = 0; k < R; ++k)
      if (8 * in_row + k * step < width) take(8 * in_row + k * step, p[k]);
    if (a.gain) {
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (8 * in_row + k * step < width) load8(a.gain, 8 * in_row + k * step, a.dim, gain[k]);
    }
  }
  if (a.norm) {
    if constexpr (R > 0) {
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (8 * in_row + k * step < width) square(p[k]);
    } else {
      for (int c = 8 * in_row; c < width; c += step) take(c, p[0]), square(p[0]);
    }
    ss = wave_sum(ss);
    if (wpr > 1) {
      if ((t & 63) == 0) part[t >> 6] = ss;
      __syncthreads();
      ss = 0.;
      for (int k = 0; k < wpr; ++k) ss += part[k];
    }
    rstd = 1. / sqrt(ss / a.dim + a.eps);
  }
  auto give = [&](int c, const Part &v, const float *g) {
    float y[8], h32[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double h = v.h(i, rr != nullptr);
      h32[i] = rr ? v.x[i] + v.res[i] : 0.f;
      y[i] = !a.norm ? v.x[i] : c + i < a.dim ? to_odd(h * rstd * (a.gain ? g[i] : 1.f)) : 0.f;
    }
    if (sr) store8(sr, c, a.dim, h32);
    store_codes8(a.out, r, c, y);
  };
  if constexpr (R > 0) {
#pragma unroll
    for (int k = 0; k < R; ++k)
      if (8 * in_row + k * step < width) give(8 * in_row + k * step, p[k], gain[k]);
  } else {
    for (int c = 8 * in_row; c < width; c += step) {
      take(c, p[0]);
      if (a.gain) load8(a.gain, c, a.dim, gain[0]);
      give(c, p[0], gain[0]);
    }
  }
}

// The values of rows in 8 bits (exact in both types)
// (`lanes` of a workgroup's 256 threads a row, a power of two)
template <typename T>
__global__ void __launch_bounds__(256) k_quant_read_rows(const RowsQuant q, int64_t n_rows, int dim, int lanes, T *out, int64_t out_stride) {
  const int64_t r = static_cast<int64_t>(blockIdx.x) * (256 / lanes) + threadIdx.x / lanes;
  if (r >= n_rows) return;
  for (int c = 8 * (threadIdx.x & (lanes - 1)); c < dim; c += 8 * lanes) {
    const uint2 w = *reinterpret_cast<const uint2 *>(q.codes + r * q.code_stride + c);
    const float s = two_to_byte(q.scale[r * q.scale_stride + c / kQuantBlock]);
    float v[8];
    dequant4(w.x, s, v), dequant4(w.y, s, v + 4);
    store8(out + r * out_stride, c, dim, v);
  }
}

// Weights in blocks of 128 by 128: one workgroup a block.  The scale is a power of two as for rows, or (a float) the largest magnitude / 448.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_weights(int n_out, int dim, const T *w, int64_t w_stride, uint8_t *codes, int64_t code_stride,
                                                       uint8_t *byte, float *scale, int64_t scale_stride) {
  __shared__ float part[4];
  const int t = threadIdx.x, c = blockIdx.x * kQuantBlock + 8 * (t & 15);
  const int64_t r0 = static_cast<int64_t>(blockIdx.y) * kQuantBlock + (t >> 4);
  float v[8][8], top = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (r0 + 16 * j < n_out) load8(w + (r0 + 16 * j) * w_stride, c, dim, v[j]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (r0 + 16 * j >= n_out) v[j][i] = 0.f;
      top = fmaxf(top, finite_mag(v[j][i]));
    }
  }
  top = wave_max(top);
  if ((t & 63) == 0) part[t >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  const float s = top > 0.f ? fmaxf(top / 448.f, 0x1p-126f) : 1.f;   // (smaller ones would lose bits of their own)
  const int e = scale_exp(top);
  const float inv = exp2_int(-e);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (r0 + 16 * j < n_out) {
      float q[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = scale ? (fabsf(v[j][i]) < INFINITY ? __builtin_amdgcn_fmed3f(v[j][i] / s, -448.f, 448.f) : NAN) : code_arg(v[j][i], inv);
      *reinterpret_cast<uint2 *>(codes + (r0 + 16 * j) * code_stride + c) = uint2{quant4(q[0], q[1], q[2], q[3]), quant4(q[4], q[5], q[6], q[7])};
    }
  if (t == 0) {
    if (scale) scale[blockIdx.y * scale_stride + blockIdx.x] = s;
    else byte[blockIdx.y * scale_stride + blockIdx.x] = static_cast<uint8_t>(e + 127);
  }
}

}  // namespace hsd
