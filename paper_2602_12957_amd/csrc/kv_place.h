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

// Last of the sequences whose first item (row or entry, by `first`) is <= x
template <typename First>
__device__ __forceinline__ int seq_by(First first, int n_seq, int x) {
  int lo = 0, hi = n_seq - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first(mid) <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Places and positions of packed rows r .. r1 - 1; `block` gives the block of a sequence's table entry.  One search a run of rows: it
// is most of what a row costs (8400 rows of 64 sequences in one workgroup 9.6 us, with a search for each 12.9).
template <typename Cu, typename Len, typename Block>
__device__ __forceinline__ void place_rows(const KvPlace &p, int r, int r1, Cu cu, Len len, Block block) {
  if (r >= r1) return;
  int s = seq_by(cu, p.n_seq, r), base = cu(s), end = cu(s + 1), S = len(s);
  for (; r < r1; ++r) {
    while (r >= end && s + 1 < p.n_seq) ++s, base = end, end = cu(s + 1), S = len(s);
    const bool mine = r < end;   // (a row behind the last sequence has no place, and position 0)
    const int pos = mine ? static_cast<int>(static_cast<uint32_t>(S) + static_cast<uint32_t>(r - base)) : 0, bi = pos / kBlk;   // (wrapped: negative)
    const int b = mine && pos >= 0 && bi < p.max_blocks ? block(s, bi) : -1;
    p.row_slot[r] = b >= 0 && b < p.n_blocks ? b * kBlk + pos % kBlk : -1;
    if (p.row_pos != nullptr) p.row_pos[r] = pos;
  }
}

// One workgroup of 1024 threads: the reservation, and the rows where there are no more than kPlaceRows.  Entries that may want a
// block are numbered through the sequences and a thread looks at every 1024th; their blocks stay in LDS for the rows.
// A chain of dependent reads: bounds, lengths and the free count; the table's entries and the top of the free stack.  16 rows 4.4 us.
constexpr int kPlaceRows = 16384, kPlaceEntries = kPlaceRows / kBlk + 2 * HSD_MAX_SEQ, kPlaceFree = 1024;
__global__ void __launch_bounds__(1024) k_kv_place(KvPlace p) {
  __shared__ int s_cu[HSD_MAX_SEQ + 1], s_len[HSD_MAX_SEQ], s_first[HSD_MAX_SEQ], s_id[kPlaceEntries], s_free[kPlaceFree], s_part[16], s_wave[16], s_flags;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const bool rows = p.total_q <= kPlaceRows;
  if (t == 0) s_flags = 0;
  const int avail = min(*p.free_count, p.n_blocks);
  for (int s = t; s <= p.n_seq; s += 1024) s_cu[s] = p.cu_q[s];
  for (int s = t; s < p.n_seq; s += 1024) s_len[s] = p.seq_len[slot_of(p.seq_slot, s, p.n_slots)];
  if (avail - 1 - t >= 0) s_free[t] = p.free_list[avail - 1 - t];   // in the order in which they are given out
  __syncthreads();
  for (int s = t; s < p.n_seq; s += 1024) {
    int bits = p.seq_slot != nullptr && p.seq_slot[s] != slot_of(p.seq_slot, s, p.n_slots) ? HSD_STATUS_BAD_SLOT : 0;
    const int S = s_len[s], n = s_cu[s + 1] - s_cu[s], lo = max(S, 0) / kBlk;
    // (sums in 64 bits: a length that no table holds is reported like one that does not fit)
    int64_t hi = n > 0 ? (static_cast<int64_t>(S) + n + kBlk - 1) / kBlk : 0;
    if (hi > p.max_blocks) bits |= HSD_STATUS_TABLE_OVERFLOW, hi = p.max_blocks;
    s_first[s] = max(static_cast<int>(hi) - lo, 0);
    if (bits) atomicOr(&s_flags, bits);
  }
  __syncthreads();
  const int entries = block_exclusive_scan_4096(s_first, p.n_seq, s_part);   // (ends with a barrier)
  // entry e of the numbering in the tables; whether it wants a block, and how many before it in its 1024 do
  auto entry = [&](int e) {
    const int s = seq_by([&](int i) { return s_first[i]; }, p.n_seq, e);
    return p.block_table + static_cast<size_t>(slot_of(p.seq_slot, s, p.n_slots)) * p.max_blocks + max(s_len[s], 0) / kBlk + (e - s_first[s]);
  };
  auto wants = [&](int e0, int32_t *&at, int &before, int &all) {
    const int e = e0 + t;
    at = e < entries ? entry(e) : nullptr;
    const int b = at != nullptr ? *at : 0;
    if (rows && at != nullptr && e < kPlaceEntries) s_id[e] = b;   // (more only if cu_q does not end at total_q)
    const bool need = b < 0;
    const unsigned long long m = __ballot(need);
    __syncthreads();   // the last round's counts have been read
    if (lane == 0) s_wave[wave] = __popcll(m);
    __syncthreads();
    before = __popcll(m & ((1ull << lane) - 1ull)), all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      const int c = s_wave[w];
      if (w < wave) before += c;
      all += c;
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
      const int rank = given + before;
      if (need) {
        const int b = rank < kPlaceFree ? s_free[rank] : p.free_list[avail - 1 - rank];
        *at = b;
        if (rows && e0 + t < kPlaceEntries) s_id[e0 + t] = b;
      }
      given += all;
    }
  }
  if (t == 0) {
    if (enough) *p.free_count = avail - total;
    const int bits = s_flags | (enough ? 0 : HSD_STATUS_POOL_EXHAUSTED);
    if (bits) atomicOr(p.status, bits);
  }
  __syncthreads();
  const int each = (p.total_q + 1023) / 1024;
  if (rows)
    place_rows(p, t * each, min((t + 1) * each, p.total_q), [&](int s) { return s_cu[s]; }, [&](int s) { return s_len[s]; },
               [&](int s, int bi) { return s_id[min(s_first[s] + bi - max(s_len[s], 0) / kBlk, kPlaceEntries - 1)]; });
}

// The rows behind the reservation, over the chip.  32772 rows of 4 sequences 11 us with the reservation.  grid: ceil(total_q / 1024), block 256
__global__ void __launch_bounds__(256) k_kv_place_rows(KvPlace p) {
  __shared__ int s_cu[HSD_MAX_SEQ + 1];
  for (int s = threadIdx.x; s <= p.n_seq; s += 256) s_cu[s] = p.cu_q[s];
  __syncthreads();
  const int r = (blockIdx.x * 256 + threadIdx.x) * 4;
  auto slot = [&](int s) { return slot_of(p.seq_slot, s, p.n_slots); };
  place_rows(p, r, min(r + 4, p.total_q), [&](int s) { return s_cu[s]; }, [&](int s) { return p.seq_len[slot(s)]; },
             [&](int s, int bi) { return p.block_table[static_cast<size_t>(slot(s)) * p.max_blocks + bi]; });
}

}  // namespace hsd
