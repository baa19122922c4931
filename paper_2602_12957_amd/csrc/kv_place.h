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

// Places and positions of packed rows t, t + step, ..; cu, state rows and lengths of the sequences by `cu`, `slot`, `len`.  Eight
// rows at a time: the search, the table entry and the stores of one row wait for one another.
template <typename Cu, typename Slot, typename Len>
__device__ __forceinline__ void place_rows(const KvPlace &p, int t, int step, Cu cu, Slot slot, Len len) {
  constexpr int U = 8;
  for (int r0 = t; r0 < p.total_q; r0 += U * step) {
    int pos[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = min(r0 + u * step, p.total_q - 1);
      int lo = 0, hi = p.n_seq - 1;   // last sequence whose first row is <= r
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cu(mid) <= r) lo = mid; else hi = mid - 1;
      }
      pos[u] = len(lo) + (r - cu(lo));
      const int bi = pos[u] / kBlk;
      b[u] = pos[u] >= 0 && bi < p.max_blocks ? p.block_table[static_cast<size_t>(slot(lo)) * p.max_blocks + bi] : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * step;
      if (r >= p.total_q) break;
      p.row_slot[r] = b[u] >= 0 && b[u] < p.n_blocks ? b[u] * kBlk + pos[u] % kBlk : -1;
      if (p.row_pos != nullptr) p.row_pos[r] = pos[u];
    }
  }
}

// One workgroup of 1024 threads: the reservation, and the rows where `rows` is set (few enough for one workgroup).
// Entries that may want a block are numbered through the sequences, and a thread looks at every 1024th.
__global__ void __launch_bounds__(1024) k_kv_place(KvPlace p, int rows) {
  __shared__ int s_cu[HSD_MAX_SEQ + 1], s_slot[HSD_MAX_SEQ], s_len[HSD_MAX_SEQ], s_first[HSD_MAX_SEQ], s_part[16], s_wave[16], s_flags;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  if (t == 0) s_flags = 0;
  const int avail = min(*p.free_count, p.n_blocks);
  for (int s = t; s <= p.n_seq; s += 1024) s_cu[s] = p.cu_q[s];
  __syncthreads();
  for (int s = t; s < p.n_seq; s += 1024) {
    const int sl = slot_of(p.seq_slot, s, p.n_slots);
    int bits = p.seq_slot != nullptr && p.seq_slot[s] != sl ? HSD_STATUS_BAD_SLOT : 0;
    const int S = p.seq_len[sl], n = s_cu[s + 1] - s_cu[s], lo = max(S, 0) / kBlk;
    int hi = n > 0 ? (S + n + kBlk - 1) / kBlk : 0;
    if (hi > p.max_blocks) bits |= HSD_STATUS_TABLE_OVERFLOW, hi = p.max_blocks;
    s_slot[s] = sl, s_len[s] = S, s_first[s] = max(hi - lo, 0);
    if (bits) atomicOr(&s_flags, bits);
  }
  __syncthreads();
  const int entries = block_exclusive_scan_4096(s_first, p.n_seq, s_part);   // (ends with a barrier)
  // entry e of the numbering: its place in the tables; whether it wants a block, and how many before it in its 1024 do
  auto entry = [&](int e) -> int32_t * {
    int lo = 0, hi = p.n_seq - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_first[mid] <= e) lo = mid; else hi = mid - 1;
    }
    return p.block_table + static_cast<size_t>(s_slot[lo]) * p.max_blocks + max(s_len[lo], 0) / kBlk + (e - s_first[lo]);
  };
  auto wants = [&](int e0, int32_t *&at, int &before, int &all) {
    const int e = e0 + t;
    at = e < entries ? entry(e) : nullptr;
    const bool need = at != nullptr && *at < 0;
    const unsigned long long m = __ballot(need);
    __syncthreads();   // the last round's counts have been read
    if (lane == 0) s_wave[wave] = __popcll(m);
    __syncthreads();
    before = __popcll(m & ((1ull << lane) - 1ull)), all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w < wave) before += s_wave[w];
      all += s_wave[w];
    }
    return need;
  };
  int32_t *at = nullptr;
  int before = 0, all = 0, total = 0;
  bool need = false;
  for (int e0 = 0; e0 < entries; e0 += 1024) {
    need = wants(e0, at, before, all);
    total += all;
  }
  const bool enough = total <= avail;
  if (enough) {
    int given = 0;
    for (int e0 = 0; e0 < entries; e0 += 1024) {
      if (entries > 1024) need = wants(e0, at, before, all);   // (one round: as it stands)
      if (need) *at = p.free_list[avail - 1 - (given + before)];
      given += all;
    }
  }
  __threadfence_block();
  __syncthreads();   // the table is complete, for this workgroup
  if (t == 0) {
    if (enough) *p.free_count = avail - total;
    const int bits = s_flags | (enough ? 0 : HSD_STATUS_POOL_EXHAUSTED);
    if (bits) atomicOr(p.status, bits);
  }
  if (rows) place_rows(p, t, 1024, [&](int s) { return s_cu[s]; }, [&](int s) { return s_slot[s]; }, [&](int s) { return s_len[s]; });
}

// The rows behind the reservation, over the chip.  grid: ceil(total_q / 2048), block 256
__global__ void __launch_bounds__(256) k_kv_place_rows(KvPlace p) {
  place_rows(p, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256, [&](int s) { return p.cu_q[s]; }, [&](int s) { return slot_of(p.seq_slot, s, p.n_slots); },
             [&](int s) { return p.seq_len[slot_of(p.seq_slot, s, p.n_slots)]; });
}

}  // namespace hsd
