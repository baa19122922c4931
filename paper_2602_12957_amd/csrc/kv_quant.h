// Keys and values held in 8 bits: pages of 16 tokens of one kv head, e4m3 codes with one power-of-two scale a page.
//
// value = code * 2^e, with e the smallest exponent for which 448 * 2^e (448: the largest code) covers the page.  With a power
// of two the scale costs no accuracy (codes are floating point: the step of a value is 2^-4 of it whatever e is, down to
// 2^-6 * 2^e), a code's value is exact in bf16, and a page whose scale has to grow (a larger token joins it) keeps the values of
// its earlier tokens but for those below 2^-6 of the new scale.  A page never holds a NaN or an infinity.
//
// Page layouts, in the order in which the attention's 32x32x16 products take their operands:
//   K  [4 sixteenths of the dims][16 tokens][16 dims]
//   V  [2 halves h][32 rows r][2 dims][8 tokens]: dims 2 r and 2 r + 1 of tokens 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3
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
// what is stored of x: finite, within the limit; `odd`: x was not finite
__device__ __forceinline__ float quant_input(float x, bool &odd) {
  odd = odd || !(fabsf(x) < INFINITY);
  return x == x ? __builtin_amdgcn_fmed3f(x, -quant_limit(), quant_limit()) : 0.f;
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

// Two and eight consecutive elements
__device__ __forceinline__ void quant_load2(const float *p, float *v) { v[0] = p[0], v[1] = p[1]; }
__device__ __forceinline__ void quant_load2(const bf16 *p, float *v) {
  typedef uint32_t u1 __attribute__((aligned(2)));
  const uint32_t x = *reinterpret_cast<const u1 *>(p);
  v[0] = __uint_as_float(x << 16), v[1] = __uint_as_float(x & 0xffff0000u);
}
__device__ __forceinline__ void quant_store2(float *p, const float *v) { p[0] = v[0], p[1] = v[1]; }
__device__ __forceinline__ void quant_store2(bf16 *p, const float *v) {
  typedef uint32_t u1 __attribute__((aligned(2)));
  *reinterpret_cast<u1 *>(p) = (__float_as_uint(v[0]) >> 16) | (__float_as_uint(v[1]) & 0xffff0000u);
}
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

// Token of the j-th byte of half vh in a V page
__device__ __forceinline__ int v_token(int j, int vh) { return 8 * (j >> 2) + 4 * vh + (j & 3); }

// Runs: rows that follow one another in one block, in the order of their slots: GAPS, slots may be left out; else they are consecutive.
// A wave looks at rows r0 .. r0 + span - 1 (span <= 16) and takes the runs that start there; one may reach 15 rows further.
template <bool GAPS>
struct RowRuns {
  int slot;                 // lane l: place of row r0 - 1 + l, l <= 32; -1 without one
  unsigned long long start; // bit l: a run starts at row r0 - 1 + l
  unsigned long long more;  // bit l: row r0 - 1 + l continues the run of the row before it
  __device__ __forceinline__ RowRuns(const int32_t *row_slot, int n_rows, int r0, int span, int n_slots, int lane) {
    const int r = r0 - 1 + lane;
    slot = lane <= 32 && r >= 0 && r < n_rows ? row_slot[r] : -1;
    if (slot >= n_slots) slot = -1;
    const int before = __shfl_up(slot, 1, kWave);
    const bool go = lane > 0 && slot >= 0 && (GAPS ? before >= 0 && before < slot && before / kBlk == slot / kBlk : slot % kBlk != 0 && before == slot - 1);
    more = __ballot(go);
    start = __ballot(lane >= 1 && lane <= span && slot >= 0 && !go);
  }
  // the first run that is left: its row, place and number of rows, and which slots of the block they are; removes it
  __device__ __forceinline__ uint32_t take(int r0, int &row, int &place, int &n) {
    const int l = __builtin_ctzll(start);
    start &= start - 1;
    row = r0 - 1 + l, place = __builtin_amdgcn_readlane(slot, l);
    n = 1 + __builtin_ctzll(~(more >> (l + 1)));
    uint32_t tokens = ((1u << n) - 1) << place % kBlk;
    if (GAPS && __builtin_amdgcn_readlane(slot, l + n - 1) != place + n - 1) {
      tokens = 0;
      for (int i = 0; i < n; ++i) tokens |= 1u << __builtin_amdgcn_readlane(slot, l + i) % kBlk;
    }
    return tokens;
  }
};
// Rows of a wave: one where that gives no more waves than the chip holds in a few rounds (a run's loads wait for one another),
// 16 beyond (a wave a row that finds no run costs its launch).  us to append, 1 / 16: 64 sequences' single tokens of 4 heads 5.0 / 41,
// 32772 rows of 4 heads 25.4 / 14.2; to read back 3.6 / 15.4 and 18.8 / 11.9.
inline int run_span(int64_t n_rows, int heads) { return n_rows * heads <= 32768 ? 1 : 16; }

// Where rows come from.  Rows of a caller, apart by strides; or a decoder pass's own, left by the projection in pages of the model's
// type (row r in page r / 16, see kv_v_elem)
template <typename T>
struct QuantRows {
  const T *k, *v;
  int64_t k_stride, v_stride;
  __device__ __forceinline__ void keys16(int r, int h, int g, float *x) const {
    const T *p = k + r * k_stride + h * kHd + 16 * g;
    quant_load8(p, x), quant_load8(p + 8, x + 8);
  }
  __device__ __forceinline__ void values2(int r, int h, int vr, float *x) const { quant_load2(v + r * v_stride + h * kHd + 2 * vr, x); }
};
template <typename T>
struct QuantStaged {
  const T *k, *v;
  int n_kv_heads;
  __device__ __forceinline__ size_t page(int r, int h) const { return (static_cast<size_t>(r / kBlk) * n_kv_heads + h) * kPageCodes; }
  __device__ __forceinline__ void keys16(int r, int h, int g, float *x) const {
    const T *p = k + page(r, h) + r % kBlk * kHd + 16 * g;
    quant_load8(p, x), quant_load8(p + 8, x + 8);
  }
  __device__ __forceinline__ void values2(int r, int h, int vr, float *x) const {
    const T *p = v + page(r, h);
    x[0] = to_f32(p[kv_v_elem(r % kBlk, 2 * vr)]), x[1] = to_f32(p[kv_v_elem(r % kBlk, 2 * vr + 1)]);
  }
};

// New rows into the pages.  One wave a run and kv head: what the page keeps of earlier tokens (slots before the run's last that are none
// of its own) and the new rows make up the page; slots behind them become 0.  A lane's 16 keys are its codes' operand order as they are, and its 8 tokens by 2
// dims of the values as well: no exchange between lanes but the page's largest magnitude.
// 32772 bf16 rows of 4 heads: 50 MB in 14.5 us, 3.5 TB/s (a large copy moves 4.9), in fp32 84 MB in 18.4; a few rows: 5 us, a chain of the places,
// the rows and the page's old codes.  (Registers bounded for twice the waves a unit: slower, the loads of a run then wait for one another.)
// grid: (ceil(n_rows / (4 * span)), n_kv_heads), block 256
template <typename Src>
__global__ void __launch_bounds__(256) k_quant_append(QuantKV kv, int n_rows, int span, const int32_t *__restrict__ row_slot, Src src,
                                                      int32_t *status) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, vh = lane >> 5, vr = lane & 31, h = blockIdx.y;
  const int r0 = (blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * span;
  if (r0 >= n_rows) return;
  RowRuns<true> runs(row_slot, n_rows, r0, span, kv.n_blocks * kBlk, lane);
  bool odd = false;
  while (runs.start != 0) {
    int r, place, n;
    const uint32_t tokens = runs.take(r0, r, place, n);
    const int last = 31 - __builtin_clz(tokens), page = place / kBlk * kv.n_kv_heads + h;
    // the run's row of a token is how many of its tokens are below
    const uint32_t high = tokens >> 4 * vh;
    const int low = __builtin_popcount(tokens & ((1u << 4 * vh) - 1));
    auto v_has = [&](int j) { return (high >> v_token(j, 0) & 1) != 0; };
    auto v_row = [&](int j) { return low + __builtin_popcount(high & ((1u << v_token(j, 0)) - 1)); };
    const bool k_has = (tokens >> c & 1) != 0;
    u32x4 *kp = reinterpret_cast<u32x4 *>(kv.k_codes + static_cast<size_t>(page) * kPageCodes) + lane;
    u32x4 *vp = reinterpret_cast<u32x4 *>(kv.v_codes + static_cast<size_t>(page) * kPageCodes) + lane;
    float kx[16], vx[8][2];   // K: dims 16 g .. of token c; V: [token v_token(j)][dim 2 vr + e]
    // (loads without a condition, of the run's nearest row where a slot is not one of its: all are in flight at once)
    src.keys16(r + min(__builtin_popcount(tokens & ((1u << c) - 1)), n - 1), h, g, kx);
#pragma unroll
    for (int j = 0; j < 8; ++j) src.values2(r + min(v_row(j), n - 1), h, vr, vx[j]);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      kx[e] = k_has ? quant_input(kx[e], odd) : 0.f;
      vx[e >> 1][e & 1] = v_has(e >> 1) ? quant_input(vx[e >> 1][e & 1], odd) : 0.f;
    }
    if (n <= last) {   // (there are slots before the last row that are not the run's)
      const u32x4 kc = *kp, vc = *vp;
      const float ks = kv.k_scale[page], vs = kv.v_scale[page];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float x[4], y[4];
        dequant4(kc[j], ks, x), dequant4(vc[j], vs, y);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (c < last && !k_has) kx[4 * j + e] = x[e];
          const int t = 4 * (j & 1) + e;
          if (v_token(t, vh) < last && !v_has(t)) vx[t][j >> 1] = y[e];
        }
      }
    }
    float ka = 0.f, va = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) ka = fmaxf(ka, fabsf(kx[e])), va = fmaxf(va, fabsf(vx[e >> 1][e & 1]));
    const int ke = scale_exp(wave_max(ka)), ve = scale_exp(wave_max(va));
    const float ki = exp2_int(-ke), vi = exp2_int(-ve);
    u32x4 kc, vc;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      kc[j] = quant4(kx[4 * j] * ki, kx[4 * j + 1] * ki, kx[4 * j + 2] * ki, kx[4 * j + 3] * ki);
      const int t = 4 * (j & 1), d = j >> 1;
      vc[j] = quant4(vx[t][d] * vi, vx[t + 1][d] * vi, vx[t + 2][d] * vi, vx[t + 3][d] * vi);
    }
    *kp = kc, *vp = vc;
    if (lane == 0) kv.k_scale[page] = exp2_int(ke), kv.v_scale[page] = exp2_int(ve);
  }
  if (status != nullptr && __any(odd) && lane == 0) atomicOr(status, HSD_STATUS_NOT_FINITE);
}

// row r's place among a pass's own rows: itself
__global__ void __launch_bounds__(256) k_own_rows(int n, int32_t *__restrict__ row) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r < n) row[r] = r;
}

// The values of rows back out of the pages; rows without a place become 0.  Runs, grid and block as for k_quant_append.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_read(QuantKV kv, int n_rows, int span, const int32_t *__restrict__ row_slot, T *__restrict__ k,
                                                    T *__restrict__ v, int64_t k_stride, int64_t v_stride) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, vh = lane >> 5, vr = lane & 31, h = blockIdx.y;
  const int r0 = (blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * span;
  if (r0 >= n_rows) return;
  RowRuns<false> runs(row_slot, n_rows, r0, span, kv.n_blocks * kBlk, lane);
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
    float kx[16], vx[8][2];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float y[4];
      dequant4(kc[j], ks, kx + 4 * j), dequant4(vc[j], vs, y);
#pragma unroll
      for (int e = 0; e < 4; ++e) vx[4 * (j & 1) + e][j >> 1] = y[e];
    }
    const int ik = c - off;
    if (ik >= 0 && ik < n) {
      T *p = k + (r + ik) * k_stride + h * kHd + 16 * g;
      quant_store8(p, kx), quant_store8(p + 8, kx + 8);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int iv = v_token(j, vh) - off;
      if (iv >= 0 && iv < n) quant_store2(v + (r + iv) * v_stride + h * kHd + 2 * vr, vx[j]);
    }
  }
}

}  // namespace hsd
