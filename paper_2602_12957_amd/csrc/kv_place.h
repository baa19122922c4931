// Rows of new tokens placed in the pages of a cache, without a pass around it: block tables extended from the free stack, and
// for every packed row its place and its position.  The same rule as a pass's own reservation (kv_reserve_block): sequence s
// takes its blocks after all sequences before it, table entries in increasing order, and where the pool is short nothing is taken.
#pragma once

#include "misc_kernels.h"

namespace hsd {

struct KvPlace {
  int n_seq, total_q, n_slots, max_blocks, n_blocks;
  const int32_t *cu_q, *seq_slot, *seq_len;
  int32_t *block_table, *free_list, *free_count, *status, *row_slot, *row_pos;
};

// Place and position of packed row r, whose sequence's bounds are looked up in `cu` (n_seq + 1 entries)
__device__ __forceinline__ void place_row(const KvPlace &p, const int32_t *cu, int r) {
  const int s = seq_of_row(cu, p.n_seq, r), sl = slot_of(p.seq_slot, s, p.n_slots);
  const int pos = p.seq_len[sl] + (r - cu[s]), bi = pos / kBlk;
  int b = -1;
  if (pos >= 0 && bi < p.max_blocks) b = p.block_table[static_cast<size_t>(sl) * p.max_blocks + bi];
  p.row_slot[r] = (b >= 0 && b < p.n_blocks) ? b * kBlk + pos % kBlk : -1;
  if (p.row_pos != nullptr) p.row_pos[r] = pos;
}

// One workgroup of 1024 threads: the reservation, and the rows where `rows` is set.
__global__ void __launch_bounds__(1024) k_kv_place(KvPlace p, int rows) {
  __shared__ int s_cnt[HSD_MAX_SEQ], s_cu[HSD_MAX_SEQ + 1], s_part[16], s_flags;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  if (t == 0) s_flags = 0;
  for (int s = t; s <= p.n_seq; s += 1024) s_cu[s] = p.cu_q[s];
  __syncthreads();
  for (int s = wave; s < p.n_seq; s += 16) {
    const int sl = slot_of(p.seq_slot, s, p.n_slots);
    if (lane == 0 && p.seq_slot != nullptr && p.seq_slot[s] != sl) atomicOr(&s_flags, HSD_STATUS_BAD_SLOT);
    const int S = p.seq_len[sl], n = s_cu[s + 1] - s_cu[s];
    int hi = n > 0 ? (S + n + kBlk - 1) / kBlk : 0;
    if (hi > p.max_blocks) {
      if (lane == 0) atomicOr(&s_flags, HSD_STATUS_TABLE_OVERFLOW);
      hi = p.max_blocks;
    }
    int cnt = 0;
    for (int i = max(S, 0) / kBlk + lane; i < hi; i += kWave) cnt += p.block_table[static_cast<size_t>(sl) * p.max_blocks + i] < 0;
    cnt = wave_sum_i(cnt);
    if (lane == 0) s_cnt[s] = cnt;
  }
  __syncthreads();
  const int total = block_exclusive_scan_4096(s_cnt, p.n_seq, s_part);
  const int avail = min(*p.free_count, p.n_blocks);
  const bool enough = total <= avail;
  if (enough) {
    for (int s = wave; s < p.n_seq; s += 16) {
      const int sl = slot_of(p.seq_slot, s, p.n_slots), S = p.seq_len[sl], n = s_cu[s + 1] - s_cu[s];
      const int hi = n > 0 ? min((S + n + kBlk - 1) / kBlk, p.max_blocks) : 0;
      int taken = s_cnt[s];
      for (int i0 = max(S, 0) / kBlk; i0 < hi; i0 += kWave) {
        const int i = i0 + lane;
        const bool need = i < hi && p.block_table[static_cast<size_t>(sl) * p.max_blocks + i] < 0;
        const unsigned long long m = __ballot(need);
        if (need) p.block_table[static_cast<size_t>(sl) * p.max_blocks + i] = p.free_list[avail - 1 - (taken + __popcll(m & ((1ull << lane) - 1ull)))];
        taken += __popcll(m);
      }
    }
  }
  __threadfence_block();
  __syncthreads();   // the table is complete, for this workgroup
  if (t == 0) {
    if (enough) *p.free_count = avail - total;
    const int bits = s_flags | (enough ? 0 : HSD_STATUS_POOL_EXHAUSTED);
    if (bits) atomicOr(p.status, bits);
  }
  if (rows)
    for (int r = t; r < p.total_q; r += 1024) place_row(p, s_cu, r);
}

}  // namespace hsd
