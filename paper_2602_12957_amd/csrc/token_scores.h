// Scores of given tokens under rows of logits: log probability, entropy of the row, its most probable tokens.
//
// The row is read once.  A thread keeps a reference m that is one of its logits, within kScoreSlack of the largest so far, and
//   Z = sum e^(x - m),   W = sum (x - m) e^(x - m)      (fp32; a -inf logit adds nothing)
// which two threads with references m, m' join as Z + Z' e^(m' - m), W + (W' + (m' - m) Z') e^(m' - m); in the end
// log p(t) = x_t - m - ln Z and the entropy is ln Z - W / Z.
//
// Alternatives.  The row's lines of 128 bytes are dealt to 64 groups in turns, and each keeps the largest value and the 16-byte piece
// in which it stands first.  The k-th largest of these 64 (value, piece) pairs bounds the k-th largest logit from below, and what
// reaches it lies in the k groups that have such a pair: only their lines are read again, k / 64 of the row.
// (Groups of single pieces read a line for each: 1856 rows of 32749 bf16 logits with eight alternatives fetched 203 MB where the
// logits are 122.)  What reaches the bound is listed in LDS (little more than k entries unless large logits lie 64 lines apart) and ranked.
//
// What bounds it: reading.  1856 bf16 rows of 32749, eight alternatives: 122 MB in 33 us, 3.7 TB/s, where a bare read reaches 6.5; 16
// fp32 rows of 32768, five: 8.2 us, what one workgroup can request at a time.
#pragma once

#include "common.h"

namespace hsd {

struct TokenScores {
  int n_rows, vocab, n_top, n_parts, part_len;   // a row in n_parts parts of part_len logits (a multiple of 64 pieces), the last shorter
  int64_t stride;
  const int32_t *tokens;
  float *logprob, *entropy, *top_logprob;
  int32_t *top_id;
  float4 *part_sums;     // [n_rows][n_parts]: m (-inf: no logit), Z, W
  uint64_t *part_top;    // [n_rows][n_parts][n_top]
};

constexpr float kScoreSlack = 8.f;   // natural orders by which a logit may exceed the reference before that moves
constexpr int kScoreList = 512;      // entries of the list in LDS

// Keys whose order is that of the alternatives: larger value first, the lower index among equals.  0: none.
__device__ __forceinline__ uint64_t score_key(float v, int i) {
  const uint32_t u = __float_as_uint(v + 0.f);   // (-0 and 0 are equal)
  const uint32_t o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return (static_cast<uint64_t>(o) << 32) | (0xffffffffu - static_cast<uint32_t>(i));
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ int key_index(uint64_t k) { return static_cast<int>(0xffffffffu - static_cast<uint32_t>(k)); }

// A piece: 16 bytes of a row, aligned to its elements
__device__ __forceinline__ u32x4 load_piece(const void *p) {
  typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
  return *reinterpret_cast<const u4 *>(p);
}
__device__ __forceinline__ void piece_values(u32x4 u, float (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(u[i]);
}
__device__ __forceinline__ void piece_values(u32x4 u, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
}
template <typename T, int E>
__device__ __forceinline__ void piece_at(const T *x, int piece, int len, float (&v)[E]) {
  const int i0 = piece * E;
  if (i0 + E <= len) {
    piece_values(load_piece(x + i0), v);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = i0 + e < len ? to_f32(x[i0 + e]) : -INFINITY;
  }
}

struct ScoreSum {
  float m, z, w;   // m: -inf where no logit was seen; z is then 0, or NaN where there was a NaN
};
// The sums of `s` with reference m (not below its own)
__device__ __forceinline__ ScoreSum score_at(const ScoreSum &s, float m) {
  if (s.m == -INFINITY) return ScoreSum{m, s.z, 0.f};
  const float d = s.m - m, f = __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
  return ScoreSum{m, s.z * f, f != 0.f ? (s.w + d * s.z) * f : 0.f};
}
// The sums of 2^n lanes together, in all of them
template <int N>
__device__ __forceinline__ ScoreSum score_lanes(ScoreSum s) {
  float m = s.m;
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
  s = score_at(s, m);
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) s.z += __shfl_xor(s.z, o, kWave), s.w += __shfl_xor(s.w, o, kWave);
  return s;
}

// What a row's sums give; v: the token's logit, -inf for none
__device__ __forceinline__ void score_write(const TokenScores &a, int r, const ScoreSum &s, bool inside, float v) {
  const float lz = logf(s.z);
  a.logprob[r] = inside && s.z != s.z ? s.z : (v == -INFINITY ? v : v - s.m - lz);
  a.entropy[r] = s.m == -INFINITY && s.z == 0.f ? 0.f : lz - s.w / s.z;
}
__device__ __forceinline__ void score_write_top(const TokenScores &a, int r, const ScoreSum &s, int rank, uint64_t key) {
  const size_t at = static_cast<size_t>(r) * a.n_top + rank;
  a.top_id[at] = key == 0 ? -1 : key_index(key);
  a.top_logprob[at] = key == 0 ? -INFINITY : key_value(key) - s.m - logf(s.z);
}

// grid: n_rows * n_parts, block 64 * NW
template <typename T, int NW>
__global__ void __launch_bounds__(64 * NW) k_token_scores(TokenScores a, const T *__restrict__ logits) {
  constexpr int E = 16 / sizeof(T), U = 4;
  // a wave's 64 pieces are 8 lines: a thread's pieces belong to NB groups, and NC waves share one
  constexpr int NB = NW < 8 ? 8 / NW : 1, NC = NW > 8 ? NW / 8 : 1;
  static_assert(U % NB == 0 && (NW % 8 == 0 || 8 % NW == 0), "a round's lines are whole turns of the groups");
  __shared__ ScoreSum s_sum[NW];
  __shared__ uint64_t s_best[NC][64], s_list[kScoreList], s_bound, s_next[NW];
  __shared__ int s_win[64], s_n, s_winners;
  const int r = blockIdx.x / a.n_parts, part = blockIdx.x - r * a.n_parts, t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
  const int first = part * a.part_len, len = min(a.part_len, a.vocab - first);
  const T *x = logits + r * a.stride + first;
  const int n_pieces = (len + E - 1) / E;
  // the token's logit, ahead of everything else
  const int tok = a.tokens[r];
  const bool inside = tok >= 0 && tok < a.vocab;
  const float tv = inside && a.n_parts == 1 ? to_f32(x[tok]) : -INFINITY;

  ScoreSum s{0.f, 0.f, 0.f};   // (m: 0 while nothing was seen, thr then -inf)
  float thr = -INFINITY, best[NB];
  int best_piece[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) best[b] = -INFINITY, best_piece[b] = 0;
  // N pieces, the first of them piece p0, the others 64 * NW apart; the first belongs to the thread's group b0
  auto take = [&](auto &v, int p0, int b0) {
    constexpr int N = sizeof(v) / sizeof(v[0]);
    float all = -INFINITY;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      float top = v[u][0];
#pragma unroll
      for (int e = 1; e < E; ++e) top = fmaxf(top, v[u][e]);
#pragma unroll
      for (int b = 0; b < NB; ++b)
        if (top > best[b] && (b0 + u) % NB == b) best[b] = top, best_piece[b] = p0 + u * 64 * NW;
      all = fmaxf(all, top);
    }
    if (all > thr) {
      const float d = s.m - all, f = thr == -INFINITY ? 0.f : expf(d);
      s.w = f != 0.f ? (s.w + d * s.z) * f : 0.f;
      s.z = thr == -INFINITY ? s.z : s.z * f;
      s.m = all, thr = all + kScoreSlack;
    }
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = v[u][e] - s.m, p = __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
        s.z += p;                                   // NaN where the logit is
        s.w = fmaf(fmaxf(d, -200.f), p, s.w);       // (below -200 p is 0)
      }
  };
  // U pieces a thread at a time, the next ones requested while these are worked on; then the pieces that are left one by one
  constexpr int kStep = 64 * NW * U;
  const int n_rounds = (len / E) / kStep;
  u32x4 raw[U];
  auto request = [&](int i) {
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = load_piece(x + static_cast<size_t>(i * kStep + u * 64 * NW + t) * E);
  };
  if (n_rounds > 0) request(0);
  for (int i = 0; i < n_rounds; ++i) {
    float v[U][E];
#pragma unroll
    for (int u = 0; u < U; ++u) piece_values(raw[u], v[u]);
    request(min(i + 1, n_rounds - 1));
    take(v, i * kStep + t, 0);
  }
  for (int p0 = n_rounds * kStep + t, b0 = 0; p0 < n_pieces; p0 += 64 * NW, ++b0) {
    float v[1][E];
    piece_at(x, p0, len, v[0]);
    take(v, p0, b0);
  }
  if (thr == -INFINITY) s.m = -INFINITY;
  s = score_lanes<64>(s);
  if (lane == 0) s_sum[wave] = s;
#pragma unroll
  for (int b = 0; b < NB; ++b) {   // the eight lanes of a line
    uint64_t key = best[b] == -INFINITY ? 0 : score_key(best[b], best_piece[b]);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1)
      key = max(key, (static_cast<uint64_t>(__shfl_xor(static_cast<uint32_t>(key >> 32), o, kWave)) << 32) |
                         static_cast<uint32_t>(__shfl_xor(static_cast<uint32_t>(key), o, kWave)));
    if ((lane & 7) == 0) s_best[wave / 8][(b * NW + wave) % 8 * 8 + (lane >> 3)] = key;
  }
  if (t == 0) s_n = 0;
  __syncthreads();
  s = score_lanes<NW>(s_sum[lane & (NW - 1)]);
  const bool whole = a.n_parts == 1;
  const size_t at = static_cast<size_t>(r) * a.n_parts + part;
  if (t == 0) {
    if (whole) score_write(a, r, s, inside, tv);
    else a.part_sums[at] = float4{s.m, s.z, s.w, 0.f};
  }
  if (a.n_top == 0) return;

  // the bound and the groups that reach it: each wave ranks 64 / NW of them
  {
    uint64_t key = s_best[0][lane];
#pragma unroll
    for (int w = 1; w < NC; ++w) key = max(key, s_best[w][lane]);
    const int n = min(__popcll(__ballot(key != 0)), a.n_top);
#pragma unroll
    for (int i = 0; i < 64 / NW; ++i) {
      const int j = wave * (64 / NW) + i;
      const uint64_t mine = (static_cast<uint64_t>(__builtin_amdgcn_readlane(static_cast<uint32_t>(key >> 32), j)) << 32) |
                            static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<uint32_t>(key), j));
      const int rank = __popcll(__ballot(key > mine));
      if (mine != 0 && rank < n) {
        s_win[rank] = j;
        if (rank == n - 1) s_bound = mine;
      }
    }
    if (t == 0) s_winners = n;
  }
  __syncthreads();
  const int winners = s_winners;
  const uint64_t bound = winners < a.n_top ? 0 : s_bound;   // fewer groups than alternatives: all their logits are listed
  // listed: keys by value and piece not behind the bound (a piece's logits have its index there, so this errs on the safe side)
  auto walk = [&](auto &&take) {
    for (int i = wave; i < winners; i += NW) {
      for (int p = 8 * (s_win[i] + 64 * (lane >> 3)) + (lane & 7); p < n_pieces; p += 8 * 64 * 8) {
        float v[E];
        piece_at(x, p, len, v);
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (v[e] > -INFINITY && score_key(v[e], p) >= bound) take(score_key(v[e], first + p * E + e));
      }
    }
  };
  walk([&](uint64_t key) {
    const int i = atomicAdd(&s_n, 1);
    if (i < kScoreList) s_list[i] = key;
  });
  __syncthreads();
  const int n = s_n;
  auto emit = [&](int rank, uint64_t key) {
    if (whole) score_write_top(a, r, s, rank, key);
    else a.part_top[at * a.n_top + rank] = key;
  };
  if (n <= kScoreList) {
    for (int i = t; i < n; i += 64 * NW) {
      const uint64_t key = s_list[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += s_list[j] > key;
      if (rank < a.n_top) emit(rank, key);
    }
    for (int i = n + t; i < a.n_top; i += 64 * NW) emit(i, 0);
    return;
  }
  // more than the list holds: one alternative after the other
  uint64_t last = ~0ull;
  for (int k = 0; k < a.n_top; ++k) {
    uint64_t mine = 0;
    walk([&](uint64_t key) {
      if (key < last && key > mine) mine = key;
    });
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t u = (static_cast<uint64_t>(__shfl_xor(static_cast<uint32_t>(mine >> 32), o, kWave)) << 32) |
                         static_cast<uint32_t>(__shfl_xor(static_cast<uint32_t>(mine), o, kWave));
      mine = max(mine, u);
    }
    if (lane == 0) s_next[wave] = mine;
    __syncthreads();
    last = s_next[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) last = max(last, s_next[w]);
    __syncthreads();
    if (t == 0) emit(k, last);
  }
}

// The parts of a row together.  grid: n_rows, block 256
constexpr int kScoreParts = 16;
template <typename T>
__global__ void __launch_bounds__(256) k_token_scores_join(TokenScores a, const T *__restrict__ logits) {
  __shared__ uint64_t s_key[kScoreParts * HSD_MAX_TOP];
  const int r = blockIdx.x, t = threadIdx.x;
  ScoreSum s{-INFINITY, 0.f, 0.f};
  if ((t & 15) < a.n_parts) {
    const float4 v = a.part_sums[static_cast<size_t>(r) * a.n_parts + (t & 15)];
    s = ScoreSum{v.x, v.y, v.z};
  }
  s = score_lanes<kScoreParts>(s);
  if (t == 0) {
    const int tok = a.tokens[r];
    const bool inside = tok >= 0 && tok < a.vocab;
    score_write(a, r, s, inside, inside ? to_f32(logits[r * a.stride + tok]) : -INFINITY);
  }
  const int n = a.n_parts * a.n_top;
  for (int i = t; i < n; i += 256) s_key[i] = a.part_top[static_cast<size_t>(r) * n + i];
  __syncthreads();
  for (int i = t; i < n; i += 256) {
    const uint64_t key = s_key[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += s_key[j] > key || (key == 0 && s_key[j] == 0 && j < i);   // (empty places in order)
    if (rank < a.n_top) score_write_top(a, r, s, rank, key);
  }
}

}  // namespace hsd
