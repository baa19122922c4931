// Keys and values held in 8 bits: pages of 16 tokens of one kv head, e4m3 codes with one power-of-two scale a page.
//
// value = code * 2^e, with e the smallest exponent for which 448 * 2^e (448: the largest code) covers the page.  With a power
// of two the scale costs no accuracy (codes are floating point: the step of a value is 2^-4 of it whatever e is, down to
// 2^-6 * 2^e), a code's value is exact in bf16, and a page whose scale has to grow (a larger token joins it) keeps the values of
// its earlier tokens but for those below 2^-6 of the new scale.  A page never holds a NaN or an infinity.
//
// Page layouts, in the order in which a wave of the attention reads them (16 bytes a lane, lane l = 16 g + c, one request a page):
//   K  lane (g, c): token c, dims 16 g .. 16 g + 15
//   V  lane (g, c): tokens 4 g .. 4 g + 3 of dim 4 c, then of dim 4 c + 1, 4 c + 2, 4 c + 3
#pragma once

#include "common.h"

namespace hsd {

constexpr int kPageCodes = kBlk * kHd;   // bytes of a page
constexpr int kScaleExpMin = -100, kScaleExpMax = 119;

struct QuantKV {
  uint8_t *k_codes, *v_codes;   // [n_blocks][n_kv_heads][1024]
  float *k_scale, *v_scale;     // [n_blocks][n_kv_heads]
  int32_t n_blocks, n_kv_heads;
};

__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }   // -126 .. 127

// Smallest e in [-100, 119] with 448 * 2^e >= amax (finite, >= 0); 0 for an empty page.  448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exp(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int x = static_cast<int>(u >> 23) - 127, e = x - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return amax > 0.f ? min(max(e, kScaleExpMin), kScaleExpMax) : 0;
}

// Largest magnitude the cache can hold: 448 * 2^119
__device__ __forceinline__ float quant_limit() { return 448.f * exp2_int(kScaleExpMax); }
// what is stored of x: finite, within the limit
__device__ __forceinline__ float quant_input(float x, bool &odd) {
  const bool nan = x != x;
  odd = odd || !(fabsf(x) <= 3.402823466e38f);
  return nan ? 0.f : fminf(fmaxf(x, -quant_limit()), quant_limit());
}
// four values of magnitude <= 448 to four e4m3 codes, nearest, ties to even
__device__ __forceinline__ uint32_t quant4(float a, float b, float c, float d) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
__device__ __forceinline__ void dequant4(uint32_t codes, float scale, float *v) {
  const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  v[0] = lo[0] * scale, v[1] = lo[1] * scale, v[2] = hi[0] * scale, v[3] = hi[1] * scale;
}

// four consecutive elements of a caller's row (aligned to its elements)
__device__ __forceinline__ void quant_load4(const float *p, float *v) {
  typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
  const f4 x = *reinterpret_cast<const f4 *>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = x[i];
}
__device__ __forceinline__ void quant_load4(const bf16 *p, float *v) {
  typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
  const u2 x = *reinterpret_cast<const u2 *>(p);
  v[0] = __uint_as_float(x[0] << 16), v[1] = __uint_as_float(x[0] & 0xffff0000u);
  v[2] = __uint_as_float(x[1] << 16), v[3] = __uint_as_float(x[1] & 0xffff0000u);
}
__device__ __forceinline__ void quant_store4(float *p, const float *v) {
  typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
  *reinterpret_cast<f4 *>(p) = f4{v[0], v[1], v[2], v[3]};
}
__device__ __forceinline__ void quant_store4(bf16 *p, const float *v) {   // (a page's values are exact in bf16)
  typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
  *reinterpret_cast<u2 *>(p) = u2{(__float_as_uint(v[0]) >> 16) | (__float_as_uint(v[1]) & 0xffff0000u),
                                  (__float_as_uint(v[2]) >> 16) | (__float_as_uint(v[3]) & 0xffff0000u)};
}

// Eight consecutive elements
__device__ __forceinline__ void quant_load8(const float *p, float *v) { quant_load4(p, v), quant_load4(p + 4, v + 4); }
__device__ __forceinline__ void quant_load8(const bf16 *p, float *v) {
  typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
  const u4 x = *reinterpret_cast<const u4 *>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(x[i] << 16), v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
}
__device__ __forceinline__ void quant_store8(float *p, const float *v) { quant_store4(p, v), quant_store4(p + 4, v + 4); }
__device__ __forceinline__ void quant_store8(bf16 *p, const float *v) {
  typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
  u4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = (__float_as_uint(v[2 * i]) >> 16) | (__float_as_uint(v[2 * i + 1]) & 0xffff0000u);
  *reinterpret_cast<u4 *>(p) = x;
}

// Runs: rows whose places are consecutive slots of one block.  A wave looks at rows r0 .. r0 + span - 1 (span <= 16) and takes
// the runs that start there; one may reach 15 rows further.
struct RowRuns {
  int slot;                 // lane l: place of row r0 - 1 + l, l <= 32; -1 without one
  unsigned long long start; // bit l: a run starts at row r0 - 1 + l
  unsigned long long more;  // bit l: row r0 - 1 + l continues the run of the row before it
  __device__ __forceinline__ RowRuns(const int32_t *row_slot, int n_rows, int r0, int span, int n_slots, int lane) {
    const int r = r0 - 1 + lane;
    slot = lane <= 32 && r >= 0 && r < n_rows ? row_slot[r] : -1;
    if (slot >= n_slots) slot = -1;
    const int before = __shfl_up(slot, 1, kWave);
    const bool go = lane > 0 && slot >= 0 && slot % kBlk != 0 && before == slot - 1;
    more = __ballot(go);
    start = __ballot(lane >= 1 && lane <= span && slot >= 0 && !go);
  }
  // the first run that is left: its row, place and number of rows; removes it
  __device__ __forceinline__ void take(int r0, int &row, int &place, int &n) {
    const int l = __builtin_ctzll(start);
    start &= start - 1;
    row = r0 - 1 + l, place = __builtin_amdgcn_readlane(slot, l);
    n = 1 + __builtin_ctzll(~(more >> (l + 1)));
  }
};
// Rows of a wave: one where that gives no more waves than the chip holds in a few rounds (a run's loads wait for one another,
// 16 runs in a row of 64 sequences' single tokens take 4 times as long), 16 beyond (a wave a row that finds no run costs its launch: 32772 rows
// of 4 heads 22.5 us against 13).
inline int run_span(int64_t n_rows, int heads) { return n_rows * heads <= 32768 ? 1 : 16; }

// New rows into the pages.  One wave a run and kv head: what the page keeps of earlier tokens (slots before the run's first) and
// the new rows make up the page; slots behind them become 0.
// grid: (ceil(n_rows / (4 * span)), n_kv_heads), block 256
template <typename T>
__global__ void __launch_bounds__(256) k_quant_append(QuantKV kv, int n_rows, int span, const int32_t *__restrict__ row_slot, const T *__restrict__ k,
                                                      const T *__restrict__ v, int64_t k_stride, int64_t v_stride, int32_t *status) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, h = blockIdx.y;
  const int r0 = (blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * span;
  if (r0 >= n_rows) return;
  RowRuns runs(row_slot, n_rows, r0, span, kv.n_blocks * kBlk, lane);
  bool odd = false;
  while (runs.start != 0) {
    int r, place, n;
    runs.take(r0, r, place, n);
    const int off = place % kBlk, page = place / kBlk * kv.n_kv_heads + h;
    u32x4 *kp = reinterpret_cast<u32x4 *>(kv.k_codes + static_cast<size_t>(page) * kPageCodes) + lane;
    u32x4 *vp = reinterpret_cast<u32x4 *>(kv.v_codes + static_cast<size_t>(page) * kPageCodes) + lane;
    float kx[16], vx[4][4];   // K: dims 16 g .. of token c; V: [token 4 g + j][dim 4 c + e]
#pragma unroll
    for (int e = 0; e < 16; ++e) kx[e] = vx[e >> 2][e & 3] = 0.f;
    const int ik = c - off;
    if (ik >= 0 && ik < n) {
      const T *p = k + (r + ik) * k_stride + h * kHd + 16 * g;
      quant_load8(p, kx), quant_load8(p + 8, kx + 8);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int iv = 4 * g + j - off;
      if (iv >= 0 && iv < n) quant_load4(v + (r + iv) * v_stride + h * kHd + 4 * c, vx[j]);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      kx[e] = quant_input(kx[e], odd);
      vx[e >> 2][e & 3] = quant_input(vx[e >> 2][e & 3], odd);
    }
    if (off > 0) {
      const u32x4 kc = *kp, vc = *vp;
      const float ks = kv.k_scale[page], vs = kv.v_scale[page];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float x[4], y[4];
        dequant4(kc[j], ks, x), dequant4(vc[j], vs, y);   // (y: dim 4 c + j of tokens 4 g ..)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (c < off) kx[4 * j + e] = x[e];
          if (4 * g + e < off) vx[e][j] = y[e];
        }
      }
    }
    float ka = 0.f, va = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) ka = fmaxf(ka, fabsf(kx[e])), va = fmaxf(va, fabsf(vx[e >> 2][e & 3]));
    const int ke = scale_exp(wave_max(ka)), ve = scale_exp(wave_max(va));
    const float ki = exp2_int(-ke), vi = exp2_int(-ve);
    u32x4 kc, vc;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      kc[j] = quant4(kx[4 * j] * ki, kx[4 * j + 1] * ki, kx[4 * j + 2] * ki, kx[4 * j + 3] * ki);
      vc[j] = quant4(vx[0][j] * vi, vx[1][j] * vi, vx[2][j] * vi, vx[3][j] * vi);
    }
    *kp = kc, *vp = vc;
    if (lane == 0) kv.k_scale[page] = exp2_int(ke), kv.v_scale[page] = exp2_int(ve);
  }
  if (status != nullptr && __any(odd) && lane == 0) atomicOr(status, HSD_STATUS_NOT_FINITE);
}

// The values of rows back out of the pages; rows without a place become 0.  Runs, grid and block as for k_quant_append.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_read(QuantKV kv, int n_rows, int span, const int32_t *__restrict__ row_slot, T *__restrict__ k,
                                                    T *__restrict__ v, int64_t k_stride, int64_t v_stride) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, h = blockIdx.y;
  const int r0 = (blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * span;
  if (r0 >= n_rows) return;
  RowRuns runs(row_slot, n_rows, r0, span, kv.n_blocks * kBlk, lane);
  unsigned long long none = __ballot(lane >= 1 && lane <= span && r0 - 1 + lane < n_rows && runs.slot < 0);
  while (none != 0) {
    const int r = r0 - 1 + __builtin_ctzll(none);
    none &= none - 1;
    k[r * k_stride + h * kHd + lane] = from_f32<T>(0.f);
    v[r * v_stride + h * kHd + lane] = from_f32<T>(0.f);
  }
  while (runs.start != 0) {
    int r, place, n;
    runs.take(r0, r, place, n);
    const int off = place % kBlk, page = place / kBlk * kv.n_kv_heads + h;
    const u32x4 kc = reinterpret_cast<const u32x4 *>(kv.k_codes + static_cast<size_t>(page) * kPageCodes)[lane];
    const u32x4 vc = reinterpret_cast<const u32x4 *>(kv.v_codes + static_cast<size_t>(page) * kPageCodes)[lane];
    const float ks = kv.k_scale[page], vs = kv.v_scale[page];
    float kx[16], vx[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float y[4];
      dequant4(kc[j], ks, kx + 4 * j), dequant4(vc[j], vs, y);
#pragma unroll
      for (int e = 0; e < 4; ++e) vx[e][j] = y[e];
    }
    const int ik = c - off;
    if (ik >= 0 && ik < n) {
      T *p = k + (r + ik) * k_stride + h * kHd + 16 * g;
      quant_store8(p, kx), quant_store8(p + 8, kx + 8);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int iv = 4 * g + j - off;
      if (iv >= 0 && iv < n) quant_store4(v + (r + iv) * v_stride + h * kHd + 4 * c, vx[j]);
    }
  }
}

}  // namespace hsd
