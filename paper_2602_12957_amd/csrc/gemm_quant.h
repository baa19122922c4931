// Products of rows and weights that are held in 8 bits, tiles of many rows.
//
//   out[m][n] = sum over blocks b of 128 columns of 2^(sa[m][b] - 127) * sw[n / 128][b] * sum_k a[m][k] w[n][k]
#pragma once

#include "rows_quant.h"

namespace hsd {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct WeightQuant {
  const uint8_t *codes;
  const void *scale;        // bytes (powers of two) or floats
  int64_t code_stride, scale_stride;
};

// N LDS-direct loads of 1 KB, N = 1, 2 or 4: lane l's 16 bytes of load j go to dst + 1024 j + 16 l; they come from base - 3 KB + off[j] + 1024 j (an
// instruction's offset moves both addresses).  In asm: the compiler would otherwise wait for every load in flight before each LDS
// read.  No register is written; the reads wait by quant_wait and a barrier.  m0 is put back as it was found.
constexpr int kLoadBias = 3 * 1024;
template <int N>
__device__ __forceinline__ void lds_load(uint32_t dst, uint64_t b, const uint32_t *off) {
  static_assert(N == 1 || N == 2 || N == 4, "loads of a group");
  uint32_t m0;   // (the base is the same in all lanes, which the compiler does not always see)
  const uint64_t p = (static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(b >> 32))) << 32) |
                     static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(b)));
  if constexpr (N == 1)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %2, %3\n\t"
                 "s_mov_b32 m0, %0" : "=&s"(m0) : "s"(dst), "v"(off[0]), "s"(p) : "memory");
  else if constexpr (N == 2)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %2, %4\n\tglobal_load_lds_dwordx4 %3, %4 offset:1024\n\t"
                 "s_mov_b32 m0, %0" : "=&s"(m0) : "s"(dst), "v"(off[0]), "v"(off[1]), "s"(p) : "memory");
  else
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %2, %6\n\tglobal_load_lds_dwordx4 %3, %6 offset:1024\n\t"
                 "global_load_lds_dwordx4 %4, %6 offset:2048\n\tglobal_load_lds_dwordx4 %5, %6 offset:%7\n\t"
                 "s_mov_b32 m0, %0" : "=&s"(m0) : "s"(dst), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(p), "n"(kLoadBias) : "memory");
}
// One of 256 bytes, 4 a lane
__device__ __forceinline__ void lds_load_256(uint32_t dst, uint64_t p) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
               "global_load_lds_dword %2, off\n\t"
               "s_mov_b32 m0, %0" : "=&s"(m0) : "s"(dst), "v"(p) : "memory");
}
// All but the N newest of this wave's loads have landed, and its LDS reads are done
template <int N>
__device__ __forceinline__ void quant_wait() {
  static_assert(N < 64, "what the counter holds");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (0 << 8) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}

// A tile of BM rows by BN weight rows, WM by WN waves; operands in a ring of S slices, each a block of 128 columns.  A step between two
// looks at LDS is half a block (H = 1) or a whole one (H = 2).  ASK: as many waves again that only request.
template <int BM_, int BN_, int WM_, int WN_, int S_, int H_ = 1, bool ASK_ = false>
struct ProductTile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NW = WM_ * WN_, S = S_, H = H_;
  static constexpr bool ASK = ASK_;
  static constexpr int TA = BM / WM / 32, TW = BN / WN / 32;      // 32x32 sub-tiles of a wave: rows, weight rows
  static constexpr int kSlice = (BM + BN) * kQuantBlock;
  static constexpr int kScales = NW * 256;                        // the rows' bytes of four blocks, in a ring of their own behind the slices
  static constexpr int kWords = (S + 3) / 4 + 1;                  // ... of so many: those of the blocks under way
  static constexpr int kLoadsA = BM / 8 / NW, kLoadsW = BN / 8 / NW, kLoads = kLoadsA + kLoadsW;   // 1 KB loads of a wave and slice
  static constexpr int kPass = TW < 2 ? TW : 2;                   // sub-tiles of columns that a wave stores at a time
  static constexpr int kRing = S * kSlice, kLds = kRing + (kWords + 1) * kScales, kThreads = 64 * NW * (ASK ? 2 : 1);
  static constexpr int out_bytes(bool gated, int size) {          // of results on their way
    return gated ? WM * 32 * (kQuantBlock + 16) + BM * WN * 4 : NW * 32 * (kPass * 32 * size + 16);
  }
  static constexpr int kGroupA = kLoadsA % 4 == 0 ? 4 : kLoadsA % 2 == 0 ? 2 : 1, kGroupW = kLoadsW % 4 == 0 ? 4 : kLoadsW % 2 == 0 ? 2 : 1;   // loads that go together
  static constexpr int kWaves = BM * BN / NW > 128 * 64 ? 1 : 2;  // of a SIMD
  static_assert(H == 1 || H == 2, "half a block or a whole one");
  static_assert(BM / 8 % NW == 0 && BN / 8 % NW == 0 && BM <= 64 * NW, "loads divide evenly");
  static_assert(S >= 2 && (S - 1) * (kLoads + 1) < 64 && kLds <= 160 * 1024, "slices in flight");
};

// Tile of a workgroup: XCD x (workgroup id mod 8) takes a contiguous run of an order that goes through bands of eight tiles of rows,
// so that the tiles an XCD works on at a time share few rows and few weights (32 of 8192^3: 8 by 4 tiles, 24 MB through its L2 a round; row after row they would take 66).
__device__ __forceinline__ void quant_tile_of(int id, int tiles_m, int tiles_n, int &tm, int &tn) {
  const int all = tiles_m * tiles_n, full = all / 8 * 8;
  const int p = id < full ? id % 8 * (full / 8) + id / 8 : id;
  const int band = p / (8 * tiles_n), rest = p - band * 8 * tiles_n, high = min(8, tiles_m - 8 * band);
  tn = rest / high;
  tm = 8 * band + rest - tn * high;
}

// silu(g) * u
__device__ __forceinline__ float swiglu(float g, float u) {
  return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g)) * u;
}

// Eight of a fragment's 32 codes as bf16, times a power of two (exact): an operand of a bf16 product
__device__ __forceinline__ bf16x8 widen(const i32x8 &f, int k, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * k], scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * k], scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * k + 1], scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * k + 1], scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A finite float scale as products take it: scale = part * 2^(byte - 127) * 2^-less, part in +-[1, 2).  `less` is to be taken from the rows' exponents, which
// are at least -100: 0 but for scales below 2^-126; a scale of 0 takes everything from them, so that all products vanish and NaN stays.  EXACT: bytes within
// 9 .. 245, so that a code times the power of two is a bf16 number.  What is missing below is taken from the rows' exponents too; what is beyond goes into part, in +-[1, 2^10) then
// (to the rows' it would make infinities of large codes, which times a code of 0 are NaN).  The sums are held divided by it: those below 2^-116 may lose bits to that.
// A scale that is no number: the byte 255, which the matrix unit takes for NaN, and with EXACT, whose codes it does not scale, the part.
struct ScaleParts {
  float part;
  uint32_t byte;
  int less;
};
template <bool EXACT>
__device__ __forceinline__ ScaleParts scale_parts(uint32_t u) {
  const uint32_t sign = u & 0x80000000u, man = u & 0x7fffffu, e = u >> 23 & 255;
  const uint32_t up = man ? __builtin_clz(man) - 8 : 0;   // to bring a subnormal one's first bit to where it is not written
  ScaleParts p;
  if (e != 0) p = {__uint_as_float(sign | 0x3f800000u | man), e, 0};
  else p = {__uint_as_float(sign | 0x3f800000u | (man << up & 0x7fffffu)), 0u, man ? static_cast<int>(up) - 1 : 255};
  if constexpr (EXACT) {
    const int b = p.byte;
    p.part = e == 255 ? NAN : __uint_as_float(__float_as_uint(p.part) + (max(b - 245, 0) << 23));
    p.byte = min(max(b, 9), 245), p.less += max(9 - b, 0);
  }
  return p;
}

// All of this wave's LDS operations are done, then those of all
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Float scales: exact products for fp32 results have a block's own sums beside the sums, added times its scale (where tiles are small that is the faster and the
// more exact: 777 rows of 1000 to 1537 8.3 us, otherwise 9.1).  With larger tiles it would take the registers of half a tile (32768 rows of 4096 to 1024 165 us, here 138):
// operands carry a scale's power of two, and the sums its rest, as ScaleParts has them: they are kept divided by that of the block at hand, so multiplied by the one before over the
// next from block to block.
//
// GATED: gate and up rows of 128 output columns (BN = 256), silu(gate) * up to 8 bits; else out.  FLOATS: weight scales are floats.
// EXACT: bf16 products of the codes instead of the 8-bit ones, by quarters of half a block (a quarter's operands are all that is in registers in 16 bits).  Grid: tiles.
template <typename Cfg, bool GATED, bool FLOATS, bool EXACT, typename T>
__global__ void __launch_bounds__(Cfg::kThreads, Cfg::kWaves) k_gemm_quant(const RowsQuant a, const WeightQuant w, int M, int N, int nk, T *__restrict__ out,
                                                                          int64_t out_stride, const RowsQuant q) {
  constexpr int BM = Cfg::BM, BN = Cfg::BN, TA = Cfg::TA, TW = Cfg::TW, NW = Cfg::NW, S = Cfg::S, H = Cfg::H;
  constexpr int COLS = GATED ? BN / 2 : BN;
  static_assert(!GATED || EXACT, "a value that becomes a code has no larger error than fp32's roundings");
  static_assert(!GATED || (COLS == kQuantBlock && TW % 2 == 0), "a workgroup has whole blocks of the rows that it rounds");
  static_assert(Cfg::out_bytes(GATED, sizeof(T)) <= Cfg::kLds, "results are staged in the operands' place");
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  const bool asks = Cfg::ASK && threadIdx.x >= 64 * NW;
  const int t = threadIdx.x - (asks ? 64 * NW : 0), lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wi = wave / Cfg::WN, wj = wave % Cfg::WN;
  int tm, tn;
  quant_tile_of(blockIdx.x, (M + BM - 1) / BM, (N + COLS - 1) / COLS, tm, tn);
  const int m0 = tm * BM, n0 = tn * COLS;

  // ---- loads.  A wave's load j of a slice covers the eight tile rows from 8 (wave kLoads + j) on (rows, and weight rows); lane l fetches, for row l / 8 of
  // them, the 16-byte piece that belongs at position l % 8: a row's pieces lie XORed by the row, so that reads of 16 rows cover all banks.
  // Rows behind the last one are that one again (their products are never stored).  Gate and up alternate by 32 rows: weight row
  // 64 g + 32 u + x of the tile is row n0 + 32 g + x of the gate or of the up projection.
  constexpr int GA = Cfg::kGroupA, GW = Cfg::kGroupW;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char *)smem_raw));
  const uint64_t base_a = reinterpret_cast<uint64_t>(a.codes) + m0 * a.code_stride - kLoadBias;
  const uint64_t base_w = reinterpret_cast<uint64_t>(w.codes) + n0 * w.code_stride - kLoadBias, up_rows = GATED ? N * w.code_stride : 0;
  uint32_t off_a[Cfg::kLoadsA], off_w[Cfg::kLoadsW];
#pragma unroll
  for (int j = 0; j < Cfg::kLoadsA; ++j) {
    const int r = (wave * Cfg::kLoadsA + j) * 8 + (lane >> 3);
    off_a[j] = min(r, M - 1 - m0) * static_cast<uint32_t>(a.code_stride) + ((lane ^ (r >> 1)) & 7) * 16 + kLoadBias - j % GA * 1024;
  }
#pragma unroll
  for (int j = 0; j < Cfg::kLoadsW; ++j) {
    const int r = (wave * Cfg::kLoadsW + j) * 8 + (lane >> 3), row = GATED ? (r >> 6) * 32 + (r & 31) : min(r, N - 1 - n0);
    off_w[j] = row * static_cast<uint32_t>(w.code_stride) + ((lane ^ (r >> 1)) & 7) * 16 + kLoadBias - j % GW * 1024;
  }
  // row t's bytes (lanes behind the tile's rows all take one word: a load's 64 lanes cost what the lines that they touch do)
  const uint64_t scales_a = reinterpret_cast<uint64_t>(a.scale) + m0 * a.scale_stride, off_s = t < BM ? min(t, M - 1 - m0) * a.scale_stride : 0;
  constexpr int LOADS = Cfg::kLoads + 1, REQUESTS = Cfg::kLoadsA / GA + Cfg::kLoadsW / GW + 1;
  auto request = [&](int kb, uint32_t place, int j) {   // request j of block kb into a slice's place
    const int col = kb * kQuantBlock;
    if (j < Cfg::kLoadsA / GA) {
      lds_load<GA>(place + (wave * Cfg::kLoadsA + j * GA) * 1024, base_a + col, off_a + j * GA);
    } else if (j < REQUESTS - 1) {
      const int k = (j - Cfg::kLoadsA / GA) * GW;
      const bool up = GATED && ((wave * Cfg::kLoadsW + k) >> 2 & 1);
      lds_load<GW>(place + BM * kQuantBlock + (wave * Cfg::kLoadsW + k) * 1024, base_w + (up ? up_rows : 0) + col, off_w + k);
    } else {
      // the rows' bytes come by words, with the first of a word's blocks; otherwise one word for all, to the place behind, so that
      // every slice has as many loads
      const bool fresh = (kb & 3) == 0;
      lds_load_256(lds0 + Cfg::kRing + (fresh ? (kb >> 2) % Cfg::kWords : Cfg::kWords) * Cfg::kScales + wave * 256,
                   scales_a + (kb & ~3) + (off_s & (fresh ? ~uint64_t{0} : 0)));
    }
  };
  constexpr int LATER = (S - 2) * LOADS;   // loads of the slices that may still be in flight when the next one is needed
  if (!Cfg::ASK || asks) {
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int j = 0; j < REQUESTS; ++j) request(min(s, nk - 1), lds0 + s * Cfg::kSlice, j);
  }
  if constexpr (Cfg::ASK) {
    if (asks) {   // passes the barriers that the others pass
      quant_wait<LATER + LOADS>();
      __builtin_amdgcn_s_barrier();
      for (int kt = 0, at = 0; kt < nk; ++kt) {
        quant_wait<LATER>();
        __builtin_amdgcn_s_barrier();
        const uint32_t place = lds0 + at * Cfg::kSlice;
        at = at + 1 == S ? 0 : at + 1;
#pragma unroll
        for (int j = 0; j < REQUESTS; ++j) request(min(kt + S, nk - 1), place, j);
      }
      quant_wait<0>();
      __builtin_amdgcn_s_barrier();
      return;
    }
  }

  // ---- scales.  The weights' come through the scalar unit, a block ahead (vector loads would be waited for with all the slices behind them).
  constexpr int kApart = FLOATS && GATED ? 2 : 1;
  uint32_t sa[kApart][TA], sa_next[TA], ws_now[2] = {0, 0}, ws_next[2] = {0, 0}, ws_byte[2];
  const int64_t wrow = GATED ? n0 : min(n0 + wj * (BN / Cfg::WN), N - 1);   // a wave's weight rows lie in one block of 128, or in one of the gate and one of up
  const int64_t ws_at[2] = {wrow / kQuantBlock * w.scale_stride, (wrow + N) / kQuantBlock * w.scale_stride};
  auto weight_scales = [&](int kb) {
#pragma unroll
    for (int i = 0; i < (GATED ? 2 : 1); ++i) {
      typedef const __attribute__((address_space(4))) uint32_t *Const;
      const uint64_t p = reinterpret_cast<uint64_t>(w.scale) + (FLOATS ? 4 : 1) * (ws_at[i] + kb);
      ws_next[i] = *reinterpret_cast<Const>(p & ~uint64_t{3});   // (a byte's word; it is looked at a block later, and so are the rows' words)
      ws_byte[i] = 8 * (p & 3);
    }
  };

  constexpr bool BLOCKS = FLOATS && EXACT && !GATED;   // a block's sums by themselves
  floatx16 acc[TW][TA], block[BLOCKS ? TW : 1][BLOCKS ? TA : 1];
  const floatx16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  // (FLOATS) what the sums are to be multiplied by, and the block's part that they are divided by; BLOCKS: what the sums of the block before are
  float factor[2] = {1.f, 1.f}, part[2] = {1.f, 1.f};
  auto rescale = [&](int i, int j) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      if constexpr (BLOCKS) acc[i][j][v] = __builtin_fmaf(block[i][j][v], factor[0], acc[i][j][v]), block[i][j][v] = 0.f;
      else acc[i][j][v] *= factor[GATED ? i & 1 : 0];
    }
  };

  // ---- fragments: row lane % 32 of a sub-tile, of its 64 bytes of a half block the 32 of lane / 32
  const int fr = lane & 31, kg = lane >> 5;
  int off_f[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) off_f[p] = fr * kQuantBlock + (((p >> 1) * 4 + kg * 2 + (p & 1)) ^ ((fr >> 1) & 7)) * 16;
  const int row_a = wi * (BM / Cfg::WM) * kQuantBlock, row_w = (BM + wj * (BN / Cfg::WN)) * kQuantBlock;
  i32x8 fa[2][H][TA], fw[2][H][TW];
  auto fragment = [&](const unsigned char *p, int half) {
    const i32x4 lo = *reinterpret_cast<const i32x4 *>(p + off_f[2 * half]), hi = *reinterpret_cast<const i32x4 *>(p + off_f[2 * half + 1]);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto read = [&](int buf, const unsigned char *p, int half, int n) {   // fragment n of a step's (weights, then rows), from half block `half` on
    const int h = n / (TA + TW), k = n % (TA + TW);
    if (k < TW) fw[buf][h][k] = fragment(p + row_w + k * 32 * kQuantBlock, half + h);
    else fa[buf][h][k - TW] = fragment(p + row_a + (k - TW) * 32 * kQuantBlock, half + h);
  };
  auto row_scales = [&](int kb) {   // words of block kb (looked at when it begins)
    const unsigned char *p = smem_raw + Cfg::kRing + (kb >> 2) % Cfg::kWords * Cfg::kScales;
#pragma unroll
    for (int i = 0; i < TA; ++i) sa_next[i] = *reinterpret_cast<const uint32_t *>(p + (wi * (BM / Cfg::WM) + i * 32 + fr) * 4);
  };
  // The products of a step, with what else it has to do dealt out between them; `begin`: it begins a block
  constexpr int PRODUCTS = TA * TW, FRAGS = H * (TA + TW), OWN = Cfg::ASK ? 0 : REQUESTS;   // (requests among the products)
  auto step = [&](int buf, bool begin, auto &&other, int others) {
    if constexpr (EXACT) {
      bf16x8 cw[TW];
#pragma unroll
      for (int n = 0; n < H * 4 * TA; ++n) {   // a quarter of half a block, of a row of sub-tiles
        const int h = n / (4 * TA), k = n / TA % 4, j = n % TA;
        if (j == 0) {
#pragma unroll
          for (int i = 0; i < TW; ++i) cw[i] = widen(fw[buf][h][i], k, BLOCKS ? 1.f : two_to_byte(ws_now[GATED ? i & 1 : 0]));
        }
        const bf16x8 ca = widen(fa[buf][h][j], k, two_to_byte(sa[0][j] & 255));
        bf16x8 cu = ca;   // (float scales may leave the rows other exponents for gate and up: next to never, but a branch here costs more than widening twice)
        if constexpr (kApart == 2) cu = widen(fa[buf][h][j], k, two_to_byte(sa[1 % kApart][j] & 255));
#pragma unroll
        for (int i = 0; i < TW; ++i) {
          if (FLOATS && begin && h == 0 && k == 0) rescale(i, j);
          floatx16 &sum = BLOCKS ? block[BLOCKS ? i : 0][BLOCKS ? j : 0] : acc[i][j];
          sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cw[i], i & 1 ? cu : ca, sum, 0, 0, 0);
        }
        for (int o = n * others / (H * TA * 4); o < (n + 1) * others / (H * TA * 4); ++o) other(o);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int n = 0; n < H * PRODUCTS; ++n) {
        const int h = n / PRODUCTS, j = n % PRODUCTS / TW, i = n % TW;
        if (FLOATS && begin && h == 0) rescale(i, j);
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fw[buf][h][i], fa[buf][h][j], acc[i][j], 0, 0, 0, ws_now[0], 0, sa[0][j]);
        for (int k = n * others / (H * PRODUCTS); k < (n + 1) * others / (H * PRODUCTS); ++k) other(k);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  // What precedes the last step of a slice: all waves have read it, and the next one is complete
  auto turn = [&]() {
    quant_wait<Cfg::ASK ? 63 : LATER>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  weight_scales(0);
  quant_wait<Cfg::ASK ? 63 : LATER + LOADS>();
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int n = 0; n < FRAGS; ++n) read(0, smem_raw, 0, n);
  row_scales(0);
  int at = 0;   // place of the slice at hand
#pragma unroll
  for (int i = 0; i < TW; ++i)
#pragma unroll
    for (int j = 0; j < TA; ++j) {
      acc[i][j] = zero;
      if constexpr (BLOCKS) block[i][j] = zero;
    }
  auto begin_block = [&](int kt) {   // scales of the block at hand, and the next one's requested
    int less[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < (GATED ? 2 : 1); ++i) {
      if constexpr (BLOCKS) {
        factor[0] = kt > 0 ? __uint_as_float(ws_now[0]) : 0.f, ws_now[0] = ws_next[0];
      } else if constexpr (FLOATS) {
        const ScaleParts p = scale_parts<EXACT>(ws_next[i]);
        factor[i] = part[i] / p.part, part[i] = p.part, ws_now[i] = p.byte, less[i] = p.less;
      } else {
        ws_now[i] = ws_next[i] >> ws_byte[i] & 255;
      }
    }
#pragma unroll
    for (int i = 0; i < TA; ++i) {
      const uint32_t x = sa_next[i] >> (8 * (kt & 3));
      sa[0][i] = FLOATS && !BLOCKS ? max(static_cast<int>(x & 255) - less[0], 0) : x;
      if constexpr (kApart == 2) sa[1][i] = max(static_cast<int>(x & 255) - less[1], 0);
    }
    weight_scales(min(kt + 1, nk - 1));
    __builtin_amdgcn_sched_barrier(0);
  };
  // Block kt; its fragments, or those of its first half, are in registers.  `u`: the set that a whole block is in.
  // (behind the last blocks the requests and reads are of the last one, or of an older one's place: nothing looks at them)
  auto do_block = [&](int kt, int u) {
    begin_block(kt);
    const unsigned char *here = smem_raw + at * Cfg::kSlice;
    const uint32_t place = lds0 + at * Cfg::kSlice;
    at = at + 1 == S ? 0 : at + 1;
    const unsigned char *next = smem_raw + at * Cfg::kSlice;
    if constexpr (H == 1) step(0, true, [&](int k) { read(1, here, 1, k); }, FRAGS);
    turn();
    const int ahead = min(kt + S, nk - 1), into = H == 1 ? 0 : u ^ 1;
    row_scales(min(kt + 1, nk - 1));
    step(H == 1 ? 1 : u, H == 2, [&](int k) { if (k < OWN) request(ahead, place, k); else read(into, next, 0, k - OWN); }, OWN + FRAGS);
  };
  if constexpr (H == 1) {
    for (int kt = 0; kt < nk; ++kt) do_block(kt, 0);
  } else {
    for (int kt = 0; kt + 1 < nk; kt += 2) do_block(kt, 0), do_block(kt + 1, 1);
    if (nk & 1) do_block(nk - 1, 0);
  }
  if constexpr (FLOATS) {
    factor[0] = BLOCKS ? __uint_as_float(ws_now[0]) : part[0], factor[1] = part[1];
#pragma unroll
    for (int i = 0; i < TW; ++i)
#pragma unroll
      for (int j = 0; j < TA; ++j) rescale(i, j);
  }
  // ---- results: lane l has row l % 32 of a sub-tile and, of its 32 weight rows, 8 (v / 4) + 4 (l / 32) + v % 4
  unsigned char *stage = smem_raw;
  quant_wait<0>();   // (of the loads that nothing looks at too: results go through the same memory)
  __builtin_amdgcn_s_barrier();
  if constexpr (!GATED) {
    // through LDS (a wave's own), so that adjacent lanes store adjacent pieces of a row
    constexpr int PASS = Cfg::kPass, W = PASS * 32, ROW = W * sizeof(T) + 16, LPR = W * sizeof(T) / 16, PER = 16 / sizeof(T);
    unsigned char *mine = stage + wave * 32 * ROW;
#pragma unroll
    for (int j = 0; j < TA; ++j)
#pragma unroll
      for (int i0 = 0; i0 < TW; i0 += PASS) {
#pragma unroll
        for (int i = 0; i < PASS; ++i)
#pragma unroll
          for (int v = 0; v < 16; v += 4) {
            T *p = reinterpret_cast<T *>(mine + fr * ROW) + i * 32 + 2 * v + 4 * kg;
            const floatx16 &x = acc[i0 + i][j];
            const floatx4 f = {x[v], x[v + 1], x[v + 2], x[v + 3]};
            if constexpr (sizeof(T) == 4) *reinterpret_cast<floatx4 *>(p) = f;
            else *reinterpret_cast<bf16x4 *>(p) = __builtin_convertvector(f, bf16x4);
          }
        const int row0 = m0 + wi * (BM / Cfg::WM) + j * 32, c0 = n0 + wj * (BN / Cfg::WN) + i0 * 32;
#pragma unroll
        for (int s = 0; s < 32 * LPR / 64; ++s) {
          const int r = s * (64 / LPR) + lane / LPR, c = lane % LPR * PER;
          const u32x4 x = *reinterpret_cast<const u32x4 *>(mine + r * ROW + lane % LPR * 16);
          if (row0 + r < M && c0 + c < N) {
            T *p = out + (row0 + r) * out_stride + c0 + c;
            if (c0 + c + PER <= N) {
              typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
              *reinterpret_cast<u4 *>(p) = x;
            } else {
              const T *y = reinterpret_cast<const T *>(mine + r * ROW + lane % LPR * 16);
              for (int k = 0; c0 + c + k < N; ++k) p[k] = y[k];
            }
          }
        }
      }
  } else {
    // 32 rows of each row of waves at a time: a row's 128 columns meet in LDS
    constexpr int P = TW / 2, ROW = kQuantBlock + 16;
    float *top = reinterpret_cast<float *>(stage + Cfg::WM * 32 * ROW);   // [BM][WN]
#pragma unroll
    for (int j = 0; j < TA; ++j) {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          acc[2 * i][j][v] = swiglu(acc[2 * i][j][v], acc[2 * i + 1][j][v]);
          m = fmaxf(m, fabsf(acc[2 * i][j][v]));
        }
      if (__builtin_expect(__any(!(m <= 448.f * 0x1p119f)), 0)) {   // infinities do not count, and what is beyond the largest scale is cut
        m = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const float y = acc[2 * i][j][v];
            m = fmaxf(m, finite_mag(y));
            acc[2 * i][j][v] = fabsf(y) < INFINITY ? __builtin_amdgcn_fmed3f(y, -448.f * 0x1p119f, 448.f * 0x1p119f) : NAN;
          }
      }
      m = half_max(m);
      if (lane < 32) top[(wi * (BM / Cfg::WM) + j * 32 + fr) * Cfg::WN + wj] = m;
    }
    lds_barrier();
#pragma unroll
    for (int j = 0; j < TA; ++j) {
      const int r = wi * (BM / Cfg::WM) + j * 32 + fr;
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < Cfg::WN; ++i) m = fmaxf(m, top[r * Cfg::WN + i]);
      const int e = scale_exp(m);
      const float inv = exp2_int(-e);
      if (j > 0) lds_barrier();   // (the rows before have been stored)
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int v = 0; v < 16; v += 4) {
          const floatx16 &y = acc[2 * i][j];
          *reinterpret_cast<uint32_t *>(stage + (wi * 32 + fr) * ROW + (wj * P + i) * 32 + 2 * v + 4 * kg) =
              quant4(y[v] * inv, y[v + 1] * inv, y[v + 2] * inv, y[v + 3] * inv);
        }
      if (wj == 0 && kg == 0 && m0 + r < M) q.scale[(m0 + r) * q.scale_stride + tn] = static_cast<uint8_t>(e + 127);
      lds_barrier();
      for (int x = t >> 3; x < 32 * Cfg::WM; x += 8 * NW) {
        const int row = m0 + (x >> 5) * (BM / Cfg::WM) + j * 32 + (x & 31);
        if (row < M) *reinterpret_cast<u32x4 *>(q.codes + row * q.code_stride + n0 + (t & 7) * 16) = *reinterpret_cast<const u32x4 *>(stage + x * ROW + (t & 7) * 16);
      }
    }
  }
}

}  // namespace hsd
