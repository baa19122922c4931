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

// A run: rows r, r + 1, .. whose places are consecutive slots of one block.  Returns the number of rows of the run that starts at
// row r, or 0 where none starts (no place, or row r - 1 is part of the same run).  All lanes of a wave alike.
__device__ __forceinline__ int run_at(const int32_t *row_slot, int n_rows, int r, int n_slots, int lane, int &slot) {
  const int i = r - 1 + lane;
  const int v = lane <= kBlk && i >= 0 && i < n_rows ? row_slot[i] : -1;
  slot = __builtin_amdgcn_readlane(v, 1);
  const int before = __builtin_amdgcn_readlane(v, 0);
  if (slot < 0 || slot >= n_slots) return 0;
  const int off = slot % kBlk;
  if (off > 0 && before == slot - 1) return 0;
  const bool ok = lane >= 1 && lane <= kBlk - off && v == slot + lane - 1;
  return __ffsll(static_cast<long long>(~(__ballot(ok) >> 1))) - 1;
}

// New rows into the pages.  One wave a run and kv head: what the page keeps of earlier tokens (slots before the run's first) and
// the new rows make up the page; slots behind them become 0.
// grid: (ceil(n_rows / 4), n_kv_heads), block 256
template <typename T>
__global__ void __launch_bounds__(256) k_quant_append(QuantKV kv, int n_rows, const int32_t *__restrict__ row_slot, const T *__restrict__ k,
                                                      const T *__restrict__ v, int64_t k_stride, int64_t v_stride, int32_t *status) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, h = blockIdx.y;
  const int r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (r >= n_rows) return;
  int slot;
  const int n = run_at(row_slot, n_rows, r, kv.n_blocks * kBlk, lane, slot);
  if (n == 0) return;
  const int off = slot % kBlk, page = slot / kBlk * kv.n_kv_heads + h;
  uint4 *kp = reinterpret_cast<uint4 *>(kv.k_codes + static_cast<size_t>(page) * kPageCodes) + lane;
  uint4 *vp = reinterpret_cast<uint4 *>(kv.v_codes + static_cast<size_t>(page) * kPageCodes) + lane;
  uint4 kc{0, 0, 0, 0}, vc{0, 0, 0, 0};
  float ks = 0.f, vs = 0.f;
  if (off > 0) kc = *kp, vc = *vp, ks = kv.k_scale[page], vs = kv.v_scale[page];
  float kx[16], vx[16];   // vx: [token][dim]
  bool odd = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    // K: dims 16 g + 4 j .. of token c
    const int i = c - off;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (i >= 0 && i < n) {
      quant_load4(k + (r + i) * k_stride + h * kHd + 16 * g + 4 * j, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = quant_input(x[e], odd);
    } else if (i < 0) {
      dequant4((&kc.x)[j], ks, x);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) kx[4 * j + e] = x[e];
    // V: token 4 g + j, dims 4 c ..
    const int iv = 4 * g + j - off;
    float y[4] = {0.f, 0.f, 0.f, 0.f};
    if (iv >= 0 && iv < n) {
      quant_load4(v + (r + iv) * v_stride + h * kHd + 4 * c, y);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = quant_input(y[e], odd);
    } else if (iv < 0) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float z[4];
        dequant4((&vc.x)[e], vs, z);
        y[e] = z[j];
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) vx[4 * j + e] = y[e];
  }
  float ka = 0.f, va = 0.f;
#pragma unroll
  for (int j = 0; j < 16; ++j) ka = fmaxf(ka, fabsf(kx[j])), va = fmaxf(va, fabsf(vx[j]));
  const int ke = scale_exp(wave_max(ka)), ve = scale_exp(wave_max(va));
  const float ki = exp2_int(-ke), vi = exp2_int(-ve);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    (&kc.x)[j] = quant4(kx[4 * j] * ki, kx[4 * j + 1] * ki, kx[4 * j + 2] * ki, kx[4 * j + 3] * ki);
    (&vc.x)[j] = quant4(vx[j] * vi, vx[4 + j] * vi, vx[8 + j] * vi, vx[12 + j] * vi);
  }
  *kp = kc, *vp = vc;
  if (lane == 0) kv.k_scale[page] = exp2_int(ke), kv.v_scale[page] = exp2_int(ve);
  if (status != nullptr && __any(odd) && lane == 0) atomicOr(status, HSD_STATUS_NOT_FINITE);
}

// The values of rows back out of the pages; rows without a place become 0.  Grid and block as k_quant_append.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_read(QuantKV kv, int n_rows, const int32_t *__restrict__ row_slot, T *__restrict__ k,
                                                    T *__restrict__ v, int64_t k_stride, int64_t v_stride) {
  const int lane = threadIdx.x & 63, h = blockIdx.y;
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= n_rows) return;
  const int slot = row_slot[r];
  float kx = 0.f, vx = 0.f;
  if (slot >= 0 && slot / kBlk < kv.n_blocks) {
    const int tok = slot % kBlk, page = slot / kBlk * kv.n_kv_heads + h;
    const size_t o = static_cast<size_t>(page) * kPageCodes;
    kx = __builtin_amdgcn_cvt_f32_fp8(kv.k_codes[o + (lane >> 4) * 256 + tok * 16 + (lane & 15)], 0) * kv.k_scale[page];
    vx = __builtin_amdgcn_cvt_f32_fp8(kv.v_codes[o + (tok >> 2) * 256 + (lane >> 2) * 16 + (lane & 3) * 4 + (tok & 3)], 0) * kv.v_scale[page];
  }
  k[r * k_stride + h * kHd + lane] = from_f32<T>(kx);
  v[r * v_stride + h * kHd + lane] = from_f32<T>(vx);
}

}  // namespace hsd
