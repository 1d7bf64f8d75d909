// Where a block of the packed-attention kernels works: which rows of which sequence, which head.
#pragma once
#include "device_common.h"
#include "kernels.h"

namespace mk {

struct PackedPlace {
  int64_t first;      // the sequence's first row
  int n, row;         // its rows; the block's first among them
  int head, kv;       // query head (the group's first where the block takes all of them), head of keys
};

// Lengths live on the device alone, so the host cannot count the row blocks.  Up to 64 sequences: a block finds its place among them
// in an order by work (packed_sorted).  More: row blocks of M rows are numbered by slots, sequence s has those from
// f(s) = ends[s-1] / M + s on.  f grows by at least ceil(rows / M) from a sequence to the next, and f(n_seq) <= T / M + n_seq: no
// table, no second launch, and at most one slot a sequence is idle.
constexpr int kPackedSorted = 64;
inline int64_t packed_slots64(int64_t T, int64_t n_seq, int M) { return T / M + n_seq; }
inline int packed_slots(int64_t T, int64_t n_seq, int M) { return (int)packed_slots64(T, n_seq, M); }
// Blocks of a launch.  Consecutive ids go to the 8 XCDs in turn.  A unit is a slot and a head of keys; its `group` query
// heads follow each other on one XCD, whose L2 then fetches the rows of keys and values once for all of them, and the
// heads of keys spread over the XCDs.
inline unsigned packed_blocks(int slots, int kv_heads, int group) { return (unsigned)((((int64_t)slots * kv_heads + 7) / 8) * 8 * group); }

// ends[s - 1], held to 0 .. T: whatever the array holds, no row outside the caller's is touched
__device__ __forceinline__ int packed_end(const PackedAttention& p, int s) { return s > 0 ? min(max(p.ends[s - 1], 0), p.T) : 0; }

template <int CTRL>
__device__ __forceinline__ int rotated(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, false); }

// Row block number `slot` of up to 64 sequences, a lane to each.  BY_WORK (behind a causal mask): those with most work first, whichever
// sequence they are of.  The row block r of a sequence of c blocks has r + 1 (own queries) or c - r (own keys) blocks to meet; so
// for each amount of work w every sequence with c >= w has one block of it, and S(w) = sum of max(0, c - w + 1) blocks have w or more:
// the block's w is the largest with S(w) > slot, by bisection.  Else the longest sequence's blocks first, which share the rows they stream.
// Against slots in the order of the rows, us: 16 causal sequences of 128-661 rows, 16 heads of 64: forward 25.2 -> 21.1, dQ 29.2 -> 25.6,
// dK/dV 45.5 -> 32.9; 6 of 1000-4096, heads of 128: 240 -> 226, 313 -> 298, 822 -> 746; fp32, 12 of 153-397 without mask: dQ 80.8 -> 74.3,
// dK/dV 107 -> 97.5.  Of 64 sequences, the most that a wave has lanes for, it gains and loses: 64 causal ones of 128-661, slots and this, forward
// and backward: 16 / 4 heads of 64 57 -> 59 and 184 -> 160, of 128 103 -> 106 and 332 -> 320; 12 / 12 of 64 49 -> 60 and 157 -> 169, fp32 422 -> 428
// and 740 -> 704.
template <int M, bool BY_WORK>
__device__ __forceinline__ bool packed_sorted(const PackedAttention& p, int slot, bool own_keys, PackedPlace& w) {
  const int lane = threadIdx.x & 63;
  const bool real = lane < p.n_seq;
  const int first = real ? packed_end(p, lane) : 0, rows = real ? max(packed_end(p, lane + 1) - first, 0) : 0, c = (rows + M - 1) / M;
  int seq, row;
  if (BY_WORK) {
    // over the wave: rows of 16 lanes by rotating sums, then their four through scalar registers
    auto total = [](int v) {
      v += rotated<0x128>(v);
      v += rotated<0x124>(v);
      v += rotated<0x122>(v);
      v += rotated<0x121>(v);
      return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) + __builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48);
    };
    int low = 1, high = c;                                   // S(low) > slot, unless there is no such block at all
    high = max(high, rotated<0x128>(high));
    high = max(high, rotated<0x124>(high));
    high = max(high, rotated<0x122>(high));
    high = max(high, rotated<0x121>(high));
    high = max(max(__builtin_amdgcn_readlane(high, 0), __builtin_amdgcn_readlane(high, 16)),
               max(__builtin_amdgcn_readlane(high, 32), __builtin_amdgcn_readlane(high, 48)));
    if (high < 1 || total(c) <= slot) return false;
    while (low < high) {
      const int mid = (low + high + 1) >> 1;
      if (total(max(0, c - mid + 1)) > slot) low = mid; else high = mid - 1;
    }
    int k = slot - total(max(0, c - low));                   // S(low + 1) blocks have more
    uint64_t with = __ballot(c >= low);
    while (k-- > 0) with &= with - 1;                        // the k-th of those that have as much
    seq = __builtin_ctzll(with);
    row = own_keys ? __builtin_amdgcn_readlane(c, seq) - low : low - 1;
  } else {
    int start = 0;                                           // blocks of the sequences before this one
    for (int i = 0; i < p.n_seq; ++i) {
      const int other = __builtin_amdgcn_readlane(c, i);
      start += other > c || (other == c && i < lane) ? other : 0;
    }
    const uint64_t mine = __ballot(start <= slot && slot < start + c);
    if (!mine) return false;
    seq = __builtin_ctzll(mine);
    row = slot - __builtin_amdgcn_readlane(start, seq);
  }
  w.first = __builtin_amdgcn_readlane(first, seq);
  w.n = __builtin_amdgcn_readlane(rows, seq);
  w.row = row * M;
  return true;
}

// the sequence of a slot: the last s with f(s) <= slot, in steps of 64
template <int M, bool CAUSAL>
__device__ __forceinline__ bool packed_rows(const PackedAttention& p, int slots, int slot, bool own_keys, PackedPlace& w) {
  if (p.n_seq <= kPackedSorted) return packed_sorted<M, CAUSAL>(p, slot, own_keys, w);
  if (!own_keys) slot = slots - 1 - slot;                    // a sequence's blocks with most work first
  const int lane = threadIdx.x & 63;
  int lo = 0, count = p.n_seq;
  while (count > 1) {
    const int stride = (count + 63) >> 6, i = lane * stride;
    const bool before = i < count && packed_end(p, lo + i) / M + lo + i <= slot;
    const int k = max(__builtin_popcountll(__ballot(before)) - 1, 0) * stride;
    lo += k;
    count = min(stride, count - k);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  const int first = __builtin_amdgcn_readfirstlane(packed_end(p, lo)), end = __builtin_amdgcn_readfirstlane(packed_end(p, lo + 1));
  w.first = first;
  w.n = end - first;
  const int64_t row = (int64_t)(slot - (first / M + lo)) * M;
  w.row = (int)row;
  return row >= 0 && row < w.n;
}

// A block of one query head; false: it has no rows.
template <int M, bool CAUSAL>
__device__ __forceinline__ bool packed_place(const PackedAttention& p, int slots, int block, PackedPlace& w) {
  const int group = p.n_heads / p.n_kv_heads, i = block >> 3;
  const int unit = i / group * 8 + (block & 7), slot = unit / p.n_kv_heads;
  if (slot >= slots) return false;
  w.kv = __builtin_amdgcn_readfirstlane(unit - slot * p.n_kv_heads);
  w.head = __builtin_amdgcn_readfirstlane(w.kv * group + i % group);
  return packed_rows<M, CAUSAL>(p, slots, __builtin_amdgcn_readfirstlane(slot), false, w);
}
// A block of all query heads of one head of keys.
template <int M, bool CAUSAL>
__device__ __forceinline__ bool packed_place_kv(const PackedAttention& p, int slots, int block, PackedPlace& w) {
  const int slot = block / p.n_kv_heads;
  if (slot >= slots) return false;
  w.kv = __builtin_amdgcn_readfirstlane(block - slot * p.n_kv_heads);
  w.head = w.kv * (p.n_heads / p.n_kv_heads);
  return packed_rows<M, CAUSAL>(p, slots, __builtin_amdgcn_readfirstlane(slot), true, w);
}

}  // namespace mk
