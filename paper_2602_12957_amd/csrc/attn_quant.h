// Attention over a cache held in 8 bits: row i of a sequence's block sees the cached tokens and rows 0 .. i of the block.
//
// One pass over the keys with a softmax reference that moves rarely.  A wave holds 32 * CT columns -- (row, query head of the kv
// head) pairs, heads fastest -- and walks pairs of pages, whose bytes are the operands of 32x32x16 products once converted to bf16
// (exact: a code times a power of two).
//   S^T = K Q^T: lane (h, c), h = lane / 32, receives keys 8 b + 4 h + e, b, e < 4, of the pair for column c
//   O^T += V^T P^T: the same lane's probabilities of a page are the operand as they are (the V pages' token order); row r of part T is
//     dim 2 r + T, so that a lane ends with dims 16 b + 8 h .. + 7, b < 4, of its column
// The row sums are 16x16x32 products with ones in half of the places, which sum both halves of each column at once: sums of the
// rounded probabilities, whose rounding cancels in the quotient.
// Probabilities in bf16 are off by half a step of 2^-8 each, which adds as much again to the rounding of the output: 2.1e-3 relative where
// that alone is 1.6e-3, and 2.4e-3 on rows that few of very many keys carry. Single tokens on caches so long that their keys are split over
// workgroups take two parts (NP), 16 bits, beside reads that they wait for anyway.
// fp32 calls split queries and probabilities into three bf16 parts each (24 bits), three products in place of one.
//
// 32x32x16 and not 16x16x32, which takes as long per product and fits 16-column decoding better: beside the short instruction the
// other wave's exponentials hardly run.  ns a wave for 36 short / 18 long ones 322 / 278, for the exponentials and what goes with
// them 271, for both, two waves a SIMD: 542 / 400.
//
// What bounds it: vector instructions, 74 a step of 32 keys by 32 columns and 16 exponentials, beside ten products: 20 of the 25 us that 16
// blocks of up to 257 rows on 1055 keys take (16 heads on 4).  Four blocks of 8193 rows on 8192 keys: 1.67 to 1.76 ms by the box, 0.94 to 0.99
// PFLOP/s, where a large product reaches 1.63.  One token of eight sequences on 131072 keys: 539 MB in 103 us and 5 to join, 5.2 TB/s, where a
// bare read reaches 6.5.  One of 64 sequences on 512 to
// 2048 keys: 13.5 us, of one 8.6: chains of four dependent reads (bounds, table, scales, codes), 3 us, and two joins' barriers.
//
// The waves of a workgroup share the columns and take every W-th pair of pages; the workgroups along grid.y take runs of
// pairs of their own where few columns would leave the chip empty (k_attn_quant_join adds them up).
#pragma once

#include "attn_wide.h"
#include "kv_quant.h"
#include "misc_kernels.h"

namespace hsd {

struct QuantAttn {
  QuantKV kv;
  int n_seq, total_q, n_slots, max_blocks, n_q_heads, group;   // group: query heads of a kv head
  const int32_t *cu_q, *seq_slot, *seq_len, *block_table;
  int64_t q_stride, o_stride;
  float scale;        // log2(e) times the softmax scale's magnitude
  uint32_t q_sign;    // its sign, to be put on the queries
  int n_tiles, n_splits;
  int heads_log;          // kv heads 1, 2, 4, 8: their logarithm; -1 for others
  uint32_t group_mul;     // x / group = x * group_mul >> kGroupShift for x < group + 64
  uint32_t waves_mul;     // x / waves = the upper half of x * waves_mul, waves > 1, x < 2^28
  float *part_o;      // [n_splits][n_tiles][n_kv_heads][columns][64]
  float2 *part_ml;    // [n_splits][n_tiles][n_kv_heads][columns]: reference, sum
};

// Quotients by what the host knows are products: a division takes some twenty instructions one after the other, and a walk of
// twelve steps had ten of them around it.  Exact: group <= 1024, so that x times what group_mul is rounded up by, group - 1 at most, stays
// below 2^22; likewise 16 waves at most and 2^32.
constexpr int kGroupShift = 22;
inline uint32_t group_mul(int group) { return ((1u << kGroupShift) + group - 1) / group; }
inline uint32_t waves_mul(int waves) { return static_cast<uint32_t>(((1ull << 32) + waves - 1) / waves); }

// Queries below 2^30, keys whose page's scale is below 2^30 (448 * 2^30 at most) and a scale below 2^50 give exponents that are
// finite.  Where one of them is not, every step looks for columns that are not: such a column's probabilities would spoil another one's row
// sum, so they are left out and the column ends as NaN.
constexpr float kCalmQuery = 0x1p30f, kCalmPage = 0x1p30f, kCalmScale = 0x1p50f;
// Common steps look at the row sums alone: above kSumMost the column's reference moves, and above kSumLost, where the products with values
// may have left the range, the walk starts again with every step a general one.
constexpr float kSumMost = 0x1p40f, kSumLost = 0x1p80f;
constexpr float kRefSlack = 20.f;          // binary orders by which a score may exceed its column's reference before that moves
// That holds for pages whose values' scale is at most kCalmValues: magnitudes below 2^47, sums of products below kSumLost times that.  A walk
// that meets a larger one takes general steps alone, without the slack, and all values 2^32 smaller: no 2^32 keys make a sum that
// overflows.  Smallest scale that an operand can be made with: 2^-126 (values below 2^-85 or so beside such a page lose bits).
constexpr float kCalmValues = 0x1p38f, kWideFactor = 0x1p-32f, kWideLeast = 0x1p-126f;
constexpr float kWideOrders = 32.f;
constexpr int kSplitPairs = 16;            // a run of pairs for a workgroup of its own is no shorter

// Tiles of `cols` columns.  Up to 64 sequences are numbered without gaps.  More: those of sequence s start at
// floor(cu_q[s] * group / cols) + s, which leaves each as many as it needs and at most one too many.
__device__ __forceinline__ int tile_start(int cu, int s, int group, int cols) { return cu * group / cols + s; }

// Sum over the lanes up to and with this one
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);    // from 1, 2, 4 and 8 lanes below in a row of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // a row's last lane to the next row, rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // lane 31 to rows 2 and 3
  return v;
}

__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

struct QuantTile {
  int slot, S, n, base, j;   // state row, cached length, rows, first packed row, tile within the sequence
};
// Sequence and place of tile t, n = 0 where there is none; by 64 lanes at a time (one round up to 64 sequences, two up to 4096)
__device__ __forceinline__ QuantTile find_tile(const QuantAttn &a, int t, int cols, int lane) {
  const bool many = a.n_seq > kWave;
  int first = 0;
  if (many) {
    const int stride = (a.n_seq + kWave - 1) / kWave, s = lane * stride;
    first = (63 - __builtin_clzll(__ballot(s < a.n_seq && tile_start(a.cu_q[min(s, a.n_seq)], s, a.group, cols) <= t))) * stride;
  }
  const int s = min(first + lane, a.n_seq - 1);
  const int cu = a.cu_q[s], end = a.cu_q[s + 1], slot = slot_of(a.seq_slot, s, a.n_slots), len = a.seq_len[slot];
  const bool in = first + lane < a.n_seq;
  const int need = in ? ((end - cu) * a.group + cols - 1) / cols : 0;
  const int start = many ? tile_start(cu, s, a.group, cols) : wave_scan(need) - need;
  // the last sequence that starts at t or before; one without rows starts where the next one does
  const unsigned long long m = __ballot(in && start <= t && (many || need > 0));
  const int hit = m != 0 ? 63 - __builtin_clzll(m) : 0;
  QuantTile q;
  q.base = __builtin_amdgcn_readlane(cu, hit);
  q.n = m != 0 ? __builtin_amdgcn_readlane(end, hit) - q.base : 0;
  q.slot = __builtin_amdgcn_readlane(slot, hit);
  // (a length that no table holds sees the whole table, as if it ended there: sums with it stay in range)
  q.S = min(max(__builtin_amdgcn_readlane(len, hit), 0), a.max_blocks * kBlk);
  q.j = t - __builtin_amdgcn_readlane(start, hit);
  return q;
}

// Workgroup b to (tile, kv head): workgroup b runs on XCD b % 8, and the tiles of one head go to as few XCDs as the heads leave it,
// so that a sequence's pages enter one or two L2s; where there are several, they take the tiles in turns (late rows see
// more keys).  Later tiles come first.  Head numbers that do not divide 8, or 8 them, keep the plain order.
__device__ __forceinline__ bool tile_of_block(const QuantAttn &a, int b, int &tile, int &h) {
  const int heads = a.kv.n_kv_heads, x = b & 7, u = b >> 3;
  int t;
  if (a.heads_log >= 0) {
    h = x & (heads - 1), t = (u << (3 - a.heads_log)) + (x >> a.heads_log);
  } else if (heads % 8 == 0) {
    h = x + 8 * (u / a.n_tiles), t = u % a.n_tiles;
  } else {
    h = b / a.n_tiles, t = b % a.n_tiles;
  }
  tile = a.n_tiles - 1 - t;
  return t < a.n_tiles && h < heads;
}
inline int heads_log(int heads) { return heads <= 8 && 8 % heads == 0 ? __builtin_ctz(heads) : -1; }
inline unsigned tile_blocks(int64_t n_tiles, int heads) {
  if (heads_log(heads) >= 0) return static_cast<unsigned>((n_tiles + 8 / heads - 1) / (8 / heads) * 8);
  return static_cast<unsigned>(n_tiles * heads);
}

// Rows and heads of a tile's columns
struct TileColumns {
  int row0, head0;   // of the first one: row of the sequence, query head of the kv head
  __device__ __forceinline__ TileColumns(const QuantAttn &a, const QuantTile &q, int cols) {
    const uint32_t f = static_cast<uint32_t>(q.j) * cols, r = f / static_cast<uint32_t>(a.group);
    row0 = scalar(static_cast<int>(r)), head0 = scalar(static_cast<int>(f - r * a.group));
  }
  __device__ __forceinline__ int row(const QuantAttn &a, int col, int &head) const {
    const uint32_t x = head0 + col, r = x * a.group_mul >> kGroupShift;
    head = static_cast<int>(x - r * a.group);
    return row0 + static_cast<int>(r);
  }
};

// Keys that the columns of a tile see, and pairs of pages of a run
__device__ __forceinline__ int tile_keys(const QuantAttn &a, const QuantTile &q, const TileColumns &tc, int cols) {
  int head;
  return scalar(min(q.S + min(tc.row(a, cols - 1, head) + 1, q.n), a.max_blocks * kBlk));
}
__device__ __forceinline__ int run_pairs(int n_pairs, int n_splits) {
  return n_splits == 1 ? max(n_pairs, kSplitPairs) : max((n_pairs + n_splits - 1) / n_splits, kSplitPairs);
}

// Eight values, four a half, as NS bf16 parts
template <int NS>
__device__ __forceinline__ void split8(const float *x, bf16x8 (&part)[NS]) {
  floatx8 f = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    part[n] = __builtin_convertvector(f, bf16x8);
    if (n + 1 < NS) f -= __builtin_convertvector(part[n], floatx8);
  }
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ bf16x8 page_operand(uint32_t a, uint32_t b, float scale) {
  const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
  const bf16x2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false), w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  return bf16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

// The largest magnitude by its bits (infinities and NaN above all numbers) of m and eight bf16 values, to the bf16 below
__device__ __forceinline__ float most_bits(float m, bf16x8 v) {
  u32x4 u = *reinterpret_cast<u32x4 *>(&v);
  uint32_t r = __float_as_uint(m);
#pragma unroll
  for (int i = 0; i < 4; ++i) r = max(r, max(u[i] & 0x7fff0000u, (u[i] << 16) & 0x7fff0000u));
  return __uint_as_float(r);
}

__device__ __forceinline__ void load_q8(const bf16 *p, uint32_t sign, bf16x8 (&part)[1]) {
  typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
  u4 u = *reinterpret_cast<const u4 *>(p);
  u ^= sign | (sign >> 16);
  part[0] = *reinterpret_cast<bf16x8 *>(&u);
}
__device__ __forceinline__ void load_q8(const float *p, uint32_t sign, bf16x8 (&part)[3]) {
  float x[8];
  quant_load4(p, x), quant_load4(p + 4, x + 4);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(__float_as_uint(x[i]) ^ sign);
  split8<3>(x, part);
}

__device__ __forceinline__ void store4(float *p, const floatx4 &v) { quant_store4(p, reinterpret_cast<const float *>(&v)); }
__device__ __forceinline__ void store4(bf16 *p, const floatx4 &v) {
  typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
  bf16x4 b = __builtin_convertvector(v, bf16x4);
  *reinterpret_cast<u2 *>(p) = *reinterpret_cast<u2 *>(&b);
}

// grid: (tile_blocks, n_splits), block 64 * W, dynamic LDS quant_attn_lds(W)
// (16 waves leave 128 registers each, which 32 bf16 columns fit; 64 columns are taken where tiles alone fill the chip: one wave.  Two of
// those fit a SIMD.  With the queries in LDS three do: 1847 us where two take 1806, four blocks of 8193 rows.)
constexpr int quant_attn_waves(bool f32, int ct) { return ct == 2 ? 1 : (f32 ? 8 : 16); }
inline int quant_attn_lds(int waves) { return waves > 1 ? waves * (64 * 32 + 64) * static_cast<int>(sizeof(float)) : 0; }

template <typename T, int CT, int NP>
__global__ void __launch_bounds__(64 * quant_attn_waves(std::is_same<T, float>::value, CT), CT == 2 ? 2 : 1) k_attn_quant(QuantAttn a, const T *__restrict__ q, T *__restrict__ out) {
  constexpr int NS = std::is_same<T, float>::value ? 3 : 1, C = 32 * CT;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int lane = threadIdx.x & 63, hf = lane >> 5, c = lane & 31;
  const int W = CT == 2 ? 1 : blockDim.x >> 6, z = blockIdx.y;
  int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  asm volatile("" : "+s"(w));   // (kept, and not made again at each use)
  int tile, h;
  if (!tile_of_block(a, blockIdx.x, tile, h)) return;
  const QuantTile qt = find_tile(a, tile, C, lane);
  const int32_t *table = a.block_table + static_cast<size_t>(qt.slot) * a.max_blocks;
  // ids of the pages of 32 steps from pair p0 on: lane 2 i + p has page p of step i
  auto page_of = [&](int pair0, int i0) { return 2 * (pair0 + w + W * (i0 + (lane >> 1))) + (lane & 1); };
  auto fetch = [&](int page) { return table[min(page, a.max_blocks - 1)]; };
  int id0 = fetch(page_of(0, 0));   // (the first ones ahead of the length where the walk starts at the first page)
  const int n_cols = qt.n * a.group - qt.j * C;   // columns from this tile's first on
  if (n_cols <= 0) return;
  const TileColumns tc(a, qt, C);
  const int n_keys = tile_keys(a, qt, tc, C), n_pages = (n_keys + kBlk - 1) / kBlk, n_pairs = (n_pages + 1) / 2;
  const int run = scalar(run_pairs(n_pairs, a.n_splits)), p0 = z * run, p1 = min(p0 + run, n_pairs);
  if (z > 0 && p0 >= p1) return;
  const bool whole = n_pairs <= run;
  const uint32_t ahead = p1 - p0 - w + W - 1;   // (a run has pairs, and w < W: not negative)
  const int n_steps = W == 1 ? ahead : scalar(static_cast<int>(__umulhi(ahead, a.waves_mul)));

  // columns
  bf16x8 qf[CT][4][NS];
  int lim[CT];   // last position that the lane's column sees
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    int hd;
    const int row = tc.row(a, min(32 * ct + c, n_cols - 1), hd);
    lim[ct] = qt.S + row;
    const T *p = q + (qt.base + row) * a.q_stride + (h * a.group + hd) * kHd + 32 * hf;
#pragma unroll
    for (int s = 0; s < 4; ++s) load_q8(p + 8 * s, a.q_sign, qf[ct][s]);
  }
  const int lim_first = qt.S + tc.row0;   // what every column sees
  float q_most = 0.f;   // (of what is no number too: the largest bits)
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int s = 0; s < 4; ++s) q_most = most_bits(q_most, qf[ct][s][0]);
  const bool calm = a.scale < kCalmScale && !__any(__float_as_uint(q_most) >= __float_as_uint(kCalmQuery));

  // Probabilities are 2^(scale s - ref).  ref is one of the column's scores, moved when one exceeds it by more than kRefSlack orders
  // (fp32 sums and bf16 probabilities have room for that), and 0 as long as the column has seen nothing.
  floatx16 o[CT][2];
  floatx4 l[CT];
  float ref[CT];
  bool seen[CT], spoilt[CT];
  bool all_seen;   // every column of the wave has
  auto clear = [&]() {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
      for (int e = 0; e < 16; ++e) o[ct][0][e] = o[ct][1][e] = 0.f;
      l[ct] = floatx4{0.f, 0.f, 0.f, 0.f};
      ref[ct] = 0.f, seen[ct] = spoilt[ct] = false;
    }
    all_seen = false;
  };
  clear();
  // As a 16x16x32 operand the lanes of columns 16 .. 31 are k groups 1 and 3 of columns 0 .. 15: rows 4 u + i sum the groups of u's parity
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = static_cast<__bf16>(((lane >> 2) & 1) == ((lane >> 4) & 1) ? 1.0f : 0.0f);

  int id = 0;
  float ksc = 1.f, vsc = 1.f;
  unsigned long long bad = 0;   // bit l: the page of lane l has no valid block
  bool wide = false;            // a page's values have a scale above kCalmValues
  auto batch = [&](int i0) {
    const int page = page_of(p0, i0);
    id = i0 == 0 && p0 == 0 ? id0 : fetch(page);
    const bool ok = page < n_pages && id >= 0 && id < a.kv.n_blocks;
    bad = __ballot(!ok);
    id = (ok ? id : 0) * a.kv.n_kv_heads + h;
    ksc = a.kv.k_scale[id], vsc = a.kv.v_scale[id];
    wide = wide || __any(ok && vsc > kCalmValues);
    if (wide) vsc = fmaxf(vsc * kWideFactor, kWideLeast);
    // they are waited for here: behind the branch around this the wait would be for every load in flight, at each step
    asm volatile("" : "+v"(id), "+v"(ksc), "+v"(vsc));
  };
  // What is in flight: the pages of the step, requested while the step before it works on its own
  u32x4 kc[2], vc[2];    // K: 32 dims of the lane's key
  struct Pages {
    uint32_t id[2];
    float ks, vs[2];
    int bad;             // bit p: page p is left out
    bool calm;
  } now, next;
  const uint8_t *k_lane = a.kv.k_codes + 512 * hf + 16 * (c & 15);
  const bool second = (c & 16) != 0;   // the lane's key is in the pair's second page
  auto request_k = [&](int i, Pages &s) {
    if ((i & 31) == 0) batch(i);
    const int src = 2 * (i & 31);
    s.bad = static_cast<int>(bad >> src) & 3;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      s.id[p] = __builtin_amdgcn_readlane(id, src + p);
      s.vs[p] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vsc), src + p));
    }
    const float ks0 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ksc), src));
    const float ks1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ksc), src + 1));
    s.ks = second ? ks1 : ks0;
    s.calm = calm && max(__float_as_uint(ks0), __float_as_uint(ks1)) < __float_as_uint(kCalmPage);
    const uint32_t id_0 = s.id[0], id_1 = s.id[1];   // (values: a choice between the members would put them into memory)
    const uint8_t *kp = k_lane + static_cast<size_t>(second ? id_1 : id_0) * kPageCodes;
    kc[0] = *reinterpret_cast<const u32x4 *>(kp), kc[1] = *reinterpret_cast<const u32x4 *>(kp + 256);
  };
  auto request_v = [&](const Pages &s) {
#pragma unroll
    for (int p = 0; p < 2; ++p) vc[p] = reinterpret_cast<const u32x4 *>(a.kv.v_codes + static_cast<size_t>(s.id[p]) * kPageCodes)[lane];
  };
  // the exponents of a step: x[ct][e] of key 8 (e / 4) + 4 hf + e % 4
  auto scores = [&](int i_next, float (&x)[CT][16]) {
    bf16x8 k[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) k[d] = page_operand(kc[d >> 1][2 * (d & 1)], kc[d >> 1][2 * (d & 1) + 1], now.ks);
    request_k(i_next, next);
    floatx16 y[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) y[ct][e] = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int n = NS - 1; n >= 0; --n) y[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[d], qf[ct][d][n], y[ct], 0, 0, 0);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[ct][e] = fmaf(y[ct][e], a.scale, -ref[ct]);
  };
  auto accumulate = [&](const float (&x)[CT][16]) {
    bf16x8 pf[CT][2][NP];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = __builtin_amdgcn_exp2f(x[ct][8 * p + e]);
        split8<NP>(y, pf[ct][p]);
      }
    bf16x8 v[2][2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int t = 0; t < 2; ++t) v[p][t] = page_operand(vc[p][2 * t], vc[p][2 * t + 1], now.vs[p]);
    request_v(next);
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int n = NP - 1; n >= 0; --n) {
          l[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[ct][p][n], l[ct], 0, 0, 0);
          o[ct][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[p][0], pf[ct][p][n], o[ct][0], 0, 0, 0);
          o[ct][1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[p][1], pf[ct][p][n], o[ct][1], 0, 0, 0);
        }
    now = next;
  };
  // A step in which keys may be hidden, references may move or columns be no numbers
  auto general = [&](int i, int i_next) {
    const int pos0 = 32 * (p0 + w + W * i);
    float x[CT][16];
    scores(i_next, x);
#pragma unroll
    for (int p = 0; p < 2; ++p)
      if ((now.bad >> p) & 1) vc[p] = u32x4{0, 0, 0, 0}, now.vs[p] = 1.f;
    bool all = true;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const int left = lim[ct] - (pos0 + 4 * hf);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (8 * (e >> 2) + (e & 3) > left || ((now.bad >> (e >> 3)) & 1) != 0) x[ct][e] = -INFINITY;
      if (!now.calm) {
        bool fine = true;
#pragma unroll
        for (int e = 0; e < 16; ++e) fine = fine && x[ct][e] < INFINITY;
        spoilt[ct] = spoilt[ct] || __shfl_xor(fine ? 0 : 1, 32, kWave) != 0 || !fine;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[ct][e] = spoilt[ct] ? -INFINITY : x[ct][e];
      }
      float m = x[ct][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) m = fmaxf(m, x[ct][e]);
      m = half_max(m);
      const bool move = m > (seen[ct] ? (wide ? 0.f : kRefSlack) : -INFINITY);
      const float by = move ? m : 0.f, f = move && seen[ct] ? __builtin_amdgcn_exp2f(-m) : 1.f;   // (nothing seen: o and l are 0)
      o[ct][0] *= f, o[ct][1] *= f, l[ct] *= f;
      ref[ct] += by, seen[ct] = seen[ct] || move;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[ct][e] -= by;
      all = all && seen[ct];
    }
    all_seen = __all(all);
    accumulate(x);
  };
  // Whether step i may be a common one: every column sees its keys and has seen some, and all is finite
  bool careful = false;
  auto common = [&](int i) { return now.bad == 0 && 32 * (p0 + w + W * i) + 31 <= lim_first && all_seen && now.calm && !careful && !wide; };
  // Whether the sums so far stand: 0, or 1 if references have to move, 2 if the walk has to start again
  // (Each half by itself: a maximum would drop a NaN, and a sum is one where the column 16 away, whose 0 it takes in, is infinite.)
  auto sums = [&]() {
    auto above = [&](float bar) {
      bool any = false;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) any = any || !(l[ct][0] <= bar);
      return __any(any) != 0;
    };
    return !above(kSumMost) ? 0 : (above(kSumLost) ? 2 : 1);
  };
  // The walk: a general step, then common ones as long as they are.  (The general one stands outside the loop over the common
  // ones: joined in one loop, their registers cost 34 moves a step.)  Pages are requested without a condition, so that no wait is
  // for more than the step's own loads.
  if (n_steps > 0) {
    const int last = n_steps - 1;
    for (int i = 0; i < n_steps;) {
      if (i == 0) {
        request_k(0, now);
        request_v(now);
        careful = careful || wide;   // (known before the first step: nothing to start again)
      }
      general(i, min(i + 1, last));
      ++i;
      int how = 0;
      while (i < n_steps && common(i) && how == 0) {
        float x[CT][16];
        scores(min(i + 1, last), x);
        accumulate(x);
        ++i;
        how = sums();
      }
      if ((how == 2 || wide) && !careful) {
        careful = true, i = 0;
        clear();
      } else if (how == 1) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
          if (l[ct][0] > kSumMost) o[ct][0] *= 1.f / kSumMost, o[ct][1] *= 1.f / kSumMost, l[ct] *= 1.f / kSumMost, ref[ct] += 40.f;
      }
    }
  }

#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    if (spoilt[ct]) l[ct][0] = __uint_as_float(0x7fc00000u);
    if (wide) l[ct][0] *= kWideFactor, ref[ct] += kWideOrders;   // (o is that much smaller already)
  }
  // the waves' parts together, four dims of a column at a time: piece i of a lane is dims 16 (i / 2) + 8 hf + 4 (i % 2) ..
  auto piece = [&](int ct, int i) {
    const int e = 4 * (i >> 1) + 2 * (i & 1);
    return floatx4{o[ct][0][e], o[ct][1][e], o[ct][0][e + 1], o[ct][1][e + 1]};
  };
  auto put = [&](int ct, int i, int ln, floatx4 x, float m, float sum) {
    const int col = 32 * ct + (ln & 31), dim = 16 * (i >> 1) + 8 * (ln >> 5) + 4 * (i & 1);
    if (col >= n_cols) return;
    if (whole) {
      int hd;
      const int row = tc.row(a, col, hd);
      x *= sum == 0.f ? 0.f : 1.f / sum;   // (of a sum of 0 all terms are)
      store4(out + (qt.base + row) * a.o_stride + (h * a.group + hd) * kHd + dim, x);
    } else {
      const size_t at = ((static_cast<size_t>(z) * a.n_tiles + tile) * a.kv.n_kv_heads + h) * C + col;
      *reinterpret_cast<floatx4 *>(a.part_o + at * kHd + dim) = x;
      if (dim == 0) a.part_ml[at] = float2{m, sum};
    }
  };
  if (W == 1) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int i = 0; i < 8; ++i) put(ct, i, lane, piece(ct, i), seen[ct] ? ref[ct] : -INFINITY, l[ct][0]);
    return;
  }
  // (32 columns: 64 are one wave's)
  float *const ml = lds + W * 2048;   // [wave][reference | sum][32]
  if (c < n_cols)   // (a token of 4 heads: 4 of the 32)
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<floatx4 *>(lds + (w * 8 + i) * 256 + lane * 4) = piece(0, i);
  if (lane < 32) {
    ml[w * 64 + lane] = seen[0] ? ref[0] : -INFINITY;
    ml[w * 64 + 32 + lane] = l[0][0];
  }
  __syncthreads();
  for (int item = threadIdx.x; item < 512; item += blockDim.x) {
    const int ln = item & 63, i = item >> 6, col = ln & 31;
    if (col >= n_cols) continue;
    float m = -INFINITY;
    for (int u = 0; u < W; ++u) m = fmaxf(m, ml[u * 64 + col]);
    const float base = m == -INFINITY ? 0.f : m;
    floatx4 x = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
    for (int u = 0; u < W; ++u) {
      const float f = __builtin_amdgcn_exp2f(ml[u * 64 + col] - base);
      x += f * *reinterpret_cast<const floatx4 *>(lds + (u * 8 + i) * 256 + ln * 4);
      sum += f * ml[u * 64 + 32 + col];
    }
    put(0, i, ln, x, m, sum);
  }
}

// The runs of a tile together, in a fixed order.  grid: (n_tiles * n_kv_heads, columns / 4), block 256: each wave takes four
// columns, 16 lanes a column, and every fourth run.
constexpr int kMaxSplits = 256;
template <typename T>
__global__ void __launch_bounds__(256) k_attn_quant_join(QuantAttn a, int cols, T *__restrict__ out) {
  __shared__ float s_f[4][kMaxSplits];
  __shared__ floatx4 s_o[4][64];
  const int h = blockIdx.x / a.n_tiles, tile = blockIdx.x % a.n_tiles, lane = threadIdx.x & 63, i = lane & 15, lc = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const QuantTile qt = find_tile(a, tile, cols, lane);
  const int n_cols = qt.n * a.group - qt.j * cols, col = blockIdx.y * 4 + lc;
  if (static_cast<int>(blockIdx.y) * 4 >= n_cols) return;
  const TileColumns tc(a, qt, cols);
  const int n_pairs = ((tile_keys(a, qt, tc, cols) + kBlk - 1) / kBlk + 1) / 2, run = run_pairs(n_pairs, a.n_splits);
  if (n_pairs <= run) return;   // written already
  const int n = (n_pairs + run - 1) / run;
  const size_t step = static_cast<size_t>(a.n_tiles) * a.kv.n_kv_heads * cols;
  const size_t at = (static_cast<size_t>(tile) * a.kv.n_kv_heads + h) * cols + min(col, n_cols - 1);
  // a lane looks at every 16th run; every wave for itself, the factors written by all alike
  float m = -INFINITY, sum = 0.f;
  for (int z = i; z < n; z += 16) m = fmaxf(m, a.part_ml[at + z * step].x);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
  const float base = m == -INFINITY ? 0.f : m;
  for (int z = i; z < n; z += 16) {
    const float2 ml = a.part_ml[at + z * step];
    const float f = exp2f(ml.x - base);
    s_f[lc][z] = f;
    sum += f * ml.y;
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
  __syncthreads();
  floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int z = w; z < n; z += 4) x += s_f[lc][z] * *reinterpret_cast<const floatx4 *>(a.part_o + (at + z * step) * kHd + 4 * i);
  s_o[w][lane] = x;
  __syncthreads();
  if (w != 0 || col >= n_cols) return;
  x = (s_o[0][lane] + s_o[1][lane]) + (s_o[2][lane] + s_o[3][lane]);
  x *= sum == 0.f ? 0.f : 1.f / sum;
  int hd;
  const int row = tc.row(a, col, hd);
  store4(out + (qt.base + row) * a.o_stride + (h * a.group + hd) * kHd + 4 * i, x);
}

}  // namespace hsd
