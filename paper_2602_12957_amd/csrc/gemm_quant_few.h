// Products of few rows (up to 64) with weights in 8 bits: bound by reading the weights, and by the way from the first request to the last sum.
//
// A workgroup has 16 weight rows; its waves share out the blocks of 128 columns (with few rows there are few workgroups: K is
// what can be split without a second launch).  Each wave brings its blocks, weights and rows, into LDS of its own, whole lines at a time,
// S of them on their way at once, and waits for nobody; the waves' sums are joined in LDS at the end, in their order.
// (Straight into registers the lanes of a load would each touch another row: 16 x 1024 from 4096 columns 11.1 us.)
#pragma once

#include "gemm_quant.h"

namespace hsd {

template <int MT>
struct FewRows {
  static constexpr int kBlock = (16 + 16 * MT) * kQuantBlock + 256;   // weights, rows, and the rows' bytes of four blocks
  static constexpr int kSlots = 2;                                    // blocks of a wave in LDS
  static constexpr int kMostWaves = MT == 1 ? 16 : 160 * 1024 / (kSlots * kBlock) > 8 ? 8 : 160 * 1024 / (kSlots * kBlock);
};

// MT: pieces of 16 rows.  Workgroup x has columns 16 x ... 16 x + 15.  EXACT: codes become bf16 (with their powers of two, exactly) for
// four 16x16x32 products instead of one 16x16x128.
template <bool FLOATS, bool EXACT, int MT, typename T>
__global__ void __launch_bounds__(64 * FewRows<MT>::kMostWaves) k_gemm_quant_few(const RowsQuant a, const WeightQuant w, int M, int N, int nk, T *__restrict__ out,
                                                                                 int64_t out_stride) {
  using Few = FewRows<MT>;
  constexpr int S = Few::kSlots, LOADS = 2 + 2 * MT + 1;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), waves = blockDim.x >> 6, l16 = lane & 15, g = lane >> 4;
  const int64_t n0 = blockIdx.x * 16;   // first weight row

  // ---- loads: 8 rows of a block each, lane l the piece of row l / 8 that belongs at l % 8 (pieces lie XORed by the row, so that
  // reads of 16 rows cover all banks).  Rows behind the last one are that one again, and not stored.
  unsigned char *mine = smem_raw + wave * S * Few::kBlock;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char *)mine));
  const uint64_t base_w = reinterpret_cast<uint64_t>(w.codes) + n0 * w.code_stride - kLoadBias, base_a = reinterpret_cast<uint64_t>(a.codes) - kLoadBias;
  uint32_t off_w[2], off_a[2 * MT];
#pragma unroll
  for (int j = 0; j < 2 + 2 * MT; ++j) {
    const int r = (j < 2 ? 8 * j : 8 * j - 16) + (lane >> 3);
    const uint32_t piece = ((lane ^ (r >> 1)) & 7) * 16;
    if (j < 2) off_w[j] = min(static_cast<int64_t>(r), N - 1 - n0) * static_cast<uint32_t>(w.code_stride) + piece + kLoadBias - j * 1024;
    else off_a[j - 2] = min(r, M - 1) * static_cast<uint32_t>(a.code_stride) + piece + kLoadBias - j % 2 * 1024;
  }
  const uint64_t scales_a = reinterpret_cast<uint64_t>(a.scale) + min(lane, M - 1) * a.scale_stride;
  auto request = [&](int kb, int slot) {
    const int b = min(kb, nk - 1), col = b * kQuantBlock;
    const uint32_t dst = lds0 + slot * Few::kBlock;
    lds_load<2>(dst, base_w + col, off_w);
#pragma unroll
    for (int j = 0; j < MT; ++j) lds_load<2>(dst + (2 + 2 * j) * 1024, base_a + col, off_a + 2 * j);
    lds_load_256(dst + (2 + 2 * MT) * 1024, scales_a + (b & ~3));
  };
  const int64_t ws_at = n0 / kQuantBlock * w.scale_stride;   // (16 weight rows lie in one block of 128)
  auto weight_scale = [&](int kb) -> uint32_t {
    typedef const __attribute__((address_space(4))) uint32_t *Const;
    const uint64_t p = reinterpret_cast<uint64_t>(w.scale) + (FLOATS ? 4 : 1) * (ws_at + min(kb, nk - 1));
    const uint32_t x = *reinterpret_cast<Const>(p & ~uint64_t{3});
    return FLOATS ? x : x >> (8 * (p & 3)) & 255;
  };

  floatx4 acc[MT];
  const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < MT; ++j) acc[j] = zero;
  const int p0 = l16 * kQuantBlock + ((2 * g) ^ (l16 >> 1)) * 16, p1 = l16 * kQuantBlock + ((2 * g + 1) ^ (l16 >> 1)) * 16;
  auto codes = [&](const unsigned char *p) {
    const i32x4 lo = *reinterpret_cast<const i32x4 *>(p + p0), hi = *reinterpret_cast<const i32x4 *>(p + p1);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  int slot = 0;
#pragma unroll
  for (int s = 0; s < S; ++s) request(wave + s * waves, s);
  for (int kb = wave; kb < nk; kb += waves) {
    const uint32_t sw = weight_scale(kb);
    quant_wait<(S - 1) * LOADS>();
    const unsigned char *b = mine + slot * Few::kBlock;
    const i32x8 cw = codes(b);
    i32x8 ca[MT];
    uint32_t sa[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      ca[j] = codes(b + (1 + j) * 2048);
      sa[j] = *reinterpret_cast<const uint32_t *>(b + (1 + MT) * 2048 + (16 * j + l16) * 4) >> (8 * (kb & 3)) & 255;
    }
    if (kb + S * waves < nk + waves) {   // (no more than one request beyond the end: the count of those in flight stays)
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      request(kb + S * waves, slot);
    }
    slot = slot + 1 == S ? 0 : slot + 1;
    bf16x8 fw[4];
    if constexpr (EXACT) {
#pragma unroll
      for (int k = 0; k < 4; ++k) fw[k] = widen(cw, k, FLOATS ? 1.f : two_to_byte(sw));
    }
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      floatx4 sum = FLOATS ? zero : acc[j];
      if constexpr (EXACT) {
#pragma unroll
        for (int k = 0; k < 4; ++k) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[k], widen(ca[j], k, two_to_byte(sa[j])), sum, 0, 0, 0);
      } else {
        sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(cw, ca[j], sum, 0, 0, 0, FLOATS ? 127 : sw, 0, sa[j]);
      }
      if constexpr (FLOATS) {
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[j][v] = __builtin_fmaf(sum[v], __uint_as_float(sw), acc[j][v]);
      } else {
        acc[j] = sum;
      }
    }
  }
  quant_wait<0>();
  __syncthreads();   // (the sums take the operands' place)

  // results: lane l has row l % 16 of a piece of rows and weight rows 4 (l / 16) + v of a piece of weights
  floatx4 *part = reinterpret_cast<floatx4 *>(smem_raw);
#pragma unroll
  for (int j = 0; j < MT; ++j) part[((wave * MT + j) * 16 + l16) * 4 + g] = acc[j];   // [wave][row][column / 4]
  __syncthreads();
  for (int x = t; x < MT * 64; x += 64 * waves) {
    floatx4 s = part[x];
    for (int k = 1; k < waves; ++k) s += part[k * MT * 64 + x];
    const int m = x / 4;
    const int64_t n = n0 + x % 4 * 4;
    if (m < M && n < N) {
      T *p = out + m * out_stride + n;
      if (n + 4 <= N) {
        const float v[4] = {s[0], s[1], s[2], s[3]};
        if constexpr (sizeof(T) == 4) {
          quant_store4(p, v);
        } else {
          typedef __bf16 b4 __attribute__((ext_vector_type(4), aligned(2)));
          *reinterpret_cast<b4 *>(p) = __builtin_convertvector(s, bf16x4);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
          if (n + k < N) p[k] = rounded<T>(s[k]);
      }
    }
  }
}

}  // namespace hsd
