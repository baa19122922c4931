// Attention over a cache held in 8 bits: row i of a sequence's block sees the cached tokens and rows 0 .. i of the block.
//
// One pass over the keys with a softmax reference that moves rarely.  A wave holds 16 * CT columns -- (row, query head of the kv
// head) pairs, heads fastest -- and walks pairs of pages: a page of K and one of V are a 16-byte request a lane each, whose bytes are
// the operands of 16x16x32 products once converted to bf16 (exact: code times a power of two).
//   S^T = K Q^T: lane (g, c) receives tokens 4 g .. 4 g + 3 of a page for column c
//   O^T += V^T P^T: the same lane's probabilities of two pages are the operand as they are; the rows of the product are dims
//     (row 4 g + i of part t: dim 16 g + 4 i + t), so that a lane ends with 16 consecutive dims of its column
// The row sums are a product with ones: sums of the rounded probabilities, whose rounding cancels in the quotient.
// fp32 calls split queries and probabilities into three bf16 parts each (24 bits), three products in place of one.
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
  float *part_o;      // [n_splits][n_tiles][n_kv_heads][columns][64]
  float2 *part_ml;    // [n_splits][n_tiles][n_kv_heads][columns]: reference, sum
};

constexpr float kRefSlack = 20.f;          // binary orders by which a score may exceed its column's reference before that moves
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
  q.S = max(__builtin_amdgcn_readlane(len, hit), 0);
  q.j = t - __builtin_amdgcn_readlane(start, hit);
  return q;
}

// Workgroup b to (tile, kv head): workgroup b runs on XCD b % 8, and the tiles of one head go to as few XCDs as the heads leave it,
// so that a sequence's pages enter one or two L2s; where there are several, they take the tiles in turns (late rows see
// more keys).  Later tiles come first.  Head numbers that do not divide 8, or 8 them, keep the plain order.
__device__ __forceinline__ bool tile_of_block(const QuantAttn &a, int b, int &tile, int &h) {
  const int heads = a.kv.n_kv_heads, x = b & 7, u = b >> 3;
  int t;
  if (heads <= 8 && 8 % heads == 0) {
    h = x % heads, t = u * (8 / heads) + x / heads;
  } else if (heads % 8 == 0) {
    h = x + 8 * (u / a.n_tiles), t = u % a.n_tiles;
  } else {
    h = b / a.n_tiles, t = b % a.n_tiles;
  }
  tile = a.n_tiles - 1 - t;
  return t < a.n_tiles && h < heads;
}
inline unsigned tile_blocks(int64_t n_tiles, int64_t heads) {
  if (heads <= 8 && 8 % heads == 0) return static_cast<unsigned>((n_tiles + 8 / heads - 1) / (8 / heads) * 8);
  return static_cast<unsigned>(n_tiles * heads);
}

// Pairs of pages that the columns of a tile see, and those of run z
__device__ __forceinline__ int tile_keys(const QuantAttn &a, const QuantTile &q, int cols) {
  return min(q.S + min(((q.j + 1) * cols - 1) / a.group + 1, q.n), a.max_blocks * kBlk);
}
__device__ __forceinline__ int run_pairs(int n_pairs, int n_splits) { return max((n_pairs + n_splits - 1) / n_splits, kSplitPairs); }

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
__device__ __forceinline__ bf16x8 page_operand(uint32_t a, uint32_t b, float sa, float sb) {
  const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, sa, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, sa, true);
  const bf16x2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, sb, false), w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, sb, true);
  return bf16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
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

// grid: (tile_blocks, n_splits), block 64 * W, dynamic LDS quant_attn_lds(W, CT)
// (16 waves leave 128 registers each, which one part of 16 bf16 columns fits)
constexpr int quant_attn_waves(bool f32, int ct) { return ct == 1 && !f32 ? 16 : 8; }
inline int quant_attn_lds(int waves, int ct) { return waves > 1 ? waves * ct * (64 * 16 + 32) * static_cast<int>(sizeof(float)) : 0; }

template <typename T, int CT>
__global__ void __launch_bounds__(64 * quant_attn_waves(std::is_same<T, float>::value, CT)) k_attn_quant(QuantAttn a, const T *__restrict__ q, T *__restrict__ out) {
  constexpr int NS = std::is_same<T, float>::value ? 3 : 1, C = 16 * CT;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int W = blockDim.x >> 6, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int z = blockIdx.y;
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
  const int n_keys = tile_keys(a, qt, C), n_pages = (n_keys + kBlk - 1) / kBlk, n_pairs = (n_pages + 1) / 2;
  const int run = run_pairs(n_pairs, a.n_splits), p0 = z * run, p1 = min(p0 + run, n_pairs);
  if (z > 0 && p0 >= p1) return;
  const bool whole = n_pairs <= run;
  const int n_steps = p1 > p0 + w ? (p1 - p0 - w + W - 1) / W : 0;

  // columns
  bf16x8 qf[CT][2][NS];
  int lim[CT];   // last position that the lane's column sees
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int f = qt.j * C + min(16 * ct + c, n_cols - 1), row = f / a.group, hd = f - row * a.group;
    lim[ct] = qt.S + row;
    const T *p = q + (qt.base + row) * a.q_stride + (h * a.group + hd) * kHd + 16 * g;
    load_q8(p, a.q_sign, qf[ct][0]);
    load_q8(p + 8, a.q_sign, qf[ct][1]);
  }
  const int lim_first = qt.S + qt.j * C / a.group;   // what every column sees

  // Probabilities are 2^(scale s - ref).  ref is one of the column's scores, moved when one exceeds it by more than kRefSlack orders
  // (fp32 sums and bf16 probabilities have room for that), and 0 as long as the column has seen nothing.
  floatx4 o[CT][4], l[CT];
  float ref[CT];
  bool seen[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
    for (int t = 0; t < 4; ++t) o[ct][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    l[ct] = floatx4{0.f, 0.f, 0.f, 0.f};
    ref[ct] = 0.f, seen[ct] = false;
  }
  bool all_seen = false;   // every column of the wave has
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = static_cast<__bf16>(1.0f);

  int id = 0;
  float ksc = 1.f, vsc = 1.f;
  unsigned long long bad = 0;   // bit l: the page of lane l has no valid block
  auto batch = [&](int i0) {
    const int page = page_of(p0, i0);
    id = i0 == 0 && p0 == 0 ? id0 : fetch(page);
    const bool ok = page < n_pages && id >= 0 && id < a.kv.n_blocks;
    bad = __ballot(!ok);
    id = (ok ? id : 0) * a.kv.n_kv_heads + h;
    ksc = a.kv.k_scale[id], vsc = a.kv.v_scale[id];
  };
  struct Step {
    u32x4 k[2], v[2];
    float ks[2], vs[2];
    int bad;   // bit p: page p is left out
  };
  auto request = [&](int i, Step &s) {
    if (i >= n_steps) return;
    if ((i & 31) == 0) batch(i);
    const int src = 2 * (i & 31);
    s.bad = static_cast<int>(bad >> src) & 3;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const size_t at = static_cast<size_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(id, src + p))) * kPageCodes;
      s.k[p] = reinterpret_cast<const u32x4 *>(a.kv.k_codes + at)[lane];
      s.v[p] = reinterpret_cast<const u32x4 *>(a.kv.v_codes + at)[lane];
      s.ks[p] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ksc), src + p));
      s.vs[p] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vsc), src + p));
    }
  };
  auto step = [&](int i, Step &s) {
    if (i >= n_steps) return;
    const int pos0 = 32 * (p0 + w + W * i);
    float x[CT][8];   // the exponents: tokens 4 g + e of the first page, then of the second
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const bf16x8 k0 = page_operand(s.k[p][0], s.k[p][1], s.ks[p], s.ks[p]), k1 = page_operand(s.k[p][2], s.k[p][3], s.ks[p], s.ks[p]);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        floatx4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = NS - 1; n >= 0; --n) {
          y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[ct][0][n], y, 0, 0, 0);
          y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[ct][1][n], y, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) x[ct][4 * p + e] = fmaf(y[e], a.scale, -ref[ct]);
      }
    }
    const bool masked = s.bad != 0 || pos0 + 31 > lim_first;
    bool move = false;   // (as integers, positive floats keep their order and negative ones lie below them)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      int m = __float_as_int(x[ct][0]);
#pragma unroll
      for (int e = 1; e < 8; ++e) m = max(m, __float_as_int(x[ct][e]));
      move = move || m > __float_as_int(kRefSlack);
    }
    if (masked || !all_seen || __any(move)) {
      if (masked) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const bool gone = (s.bad >> p) & 1;
          if (gone) s.v[p] = u32x4{0, 0, 0, 0}, s.vs[p] = 1.f;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            const int left = gone ? -1 : lim[ct] - (pos0 + 16 * p + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e > left) x[ct][4 * p + e] = -INFINITY;
          }
        }
      }
      bool all = true;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float m = x[ct][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) m = fmaxf(m, x[ct][e]);
        m = half_max(quarter_max(m));
        if (m > (seen[ct] ? kRefSlack : -INFINITY)) {
          const float f = __builtin_amdgcn_exp2f(-m);   // (nothing seen: o and l are 0 or NaN, whatever f is, unless it is inf)
#pragma unroll
          for (int t = 0; t < 4; ++t) o[ct][t] = seen[ct] ? o[ct][t] * f : o[ct][t];
          l[ct] = seen[ct] ? l[ct] * f : l[ct];
          ref[ct] += m, seen[ct] = true;
#pragma unroll
          for (int e = 0; e < 8; ++e) x[ct][e] -= m;
        }
        all = all && seen[ct];
      }
      all_seen = __all(all);
    }
    bf16x8 v[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = page_operand(s.v[0][t], s.v[1][t], s.vs[0], s.vs[1]);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(x[ct][e]);
      bf16x8 pf[NS];
      split8<NS>(p, pf);
#pragma unroll
      for (int n = NS - 1; n >= 0; --n) {
#pragma unroll
        for (int t = 0; t < 4; ++t) o[ct][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[t], pf[n], o[ct][t], 0, 0, 0);
        l[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[n], l[ct], 0, 0, 0);
      }
    }
  };
  Step s0, s1;
  request(0, s0);
  for (int i = 0; i < n_steps; i += 2) {
    request(i + 1, s1);
    step(i, s0);
    request(i + 2, s0);
    step(i + 1, s1);
  }

  // the waves' parts together; a column's 16 dims of a lane in pieces of four
  auto put = [&](int ct, int i, int ln, floatx4 x, float m, float sum) {
    const int col = 16 * ct + (ln & 15), dim = 16 * (ln >> 4) + 4 * i;
    if (col >= n_cols) return;
    if (whole) {
      const int f = qt.j * C + col, row = f / a.group, hd = f - row * a.group;
      if (sum == 0.f) x = floatx4{0.f, 0.f, 0.f, 0.f};
      else x /= sum;
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
      for (int i = 0; i < 4; ++i)
        put(ct, i, lane, floatx4{o[ct][0][i], o[ct][1][i], o[ct][2][i], o[ct][3][i]}, seen[ct] ? ref[ct] : -INFINITY, l[ct][0]);
    return;
  }
  float *const ml = lds + W * CT * 1024;   // [wave][part of 16 columns][reference | sum][16]
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<floatx4 *>(lds + ((w * CT + ct) * 4 + i) * 256 + lane * 4) = floatx4{o[ct][0][i], o[ct][1][i], o[ct][2][i], o[ct][3][i]};
    if (lane < 16) {
      ml[(w * CT + ct) * 32 + lane] = seen[ct] ? ref[ct] : -INFINITY;
      ml[(w * CT + ct) * 32 + 16 + lane] = l[ct][0];
    }
  }
  __syncthreads();
  for (int item = threadIdx.x; item < 256 * CT; item += blockDim.x) {
    const int ln = item & 63, i = (item >> 6) & 3, ct = item >> 8;
    float m = -INFINITY;
    for (int u = 0; u < W; ++u) m = fmaxf(m, ml[(u * CT + ct) * 32 + (ln & 15)]);
    const float base = m == -INFINITY ? 0.f : m;
    floatx4 x = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
    for (int u = 0; u < W; ++u) {
      const float f = exp2f(ml[(u * CT + ct) * 32 + (ln & 15)] - base);
      x += f * *reinterpret_cast<const floatx4 *>(lds + ((u * CT + ct) * 4 + i) * 256 + ln * 4);
      sum += f * ml[(u * CT + ct) * 32 + 16 + (ln & 15)];
    }
    put(ct, i, ln, x, m, sum);
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
  const int n_pairs = ((tile_keys(a, qt, cols) + kBlk - 1) / kBlk + 1) / 2, run = run_pairs(n_pairs, a.n_splits);
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
  if (sum == 0.f) x = floatx4{0.f, 0.f, 0.f, 0.f};
  else x /= sum;
  const int f = qt.j * cols + col, row = f / a.group, hd = f - row * a.group;
  store4(out + (qt.base + row) * a.o_stride + (h * a.group + hd) * kHd + 4 * i, x);
}

}  // namespace hsd
