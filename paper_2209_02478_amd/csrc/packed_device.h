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

// Row blocks of M rows are numbered by slots: sequence s has those from f(s) = ends[s-1] / M + s on.  f grows by at
// least ceil(rows / M) from a sequence to the next, and f(n_seq) <= T / M + n_seq: no table, no second launch, and at most
// one slot a sequence is idle.  Lengths live on the device alone, so the host could not count the blocks.
inline int64_t packed_slots64(int64_t T, int64_t n_seq, int M) { return T / M + n_seq; }
inline int packed_slots(int64_t T, int64_t n_seq, int M) { return (int)packed_slots64(T, n_seq, M); }
// Blocks of a launch.  Consecutive ids go to the 8 XCDs in turn.  A unit is a slot and a head of keys; its `group` query
// heads follow each other on one XCD, whose L2 then fetches the rows of keys and values once for all of them, and the
// heads of keys spread over the XCDs.
inline unsigned packed_blocks(int slots, int kv_heads, int group) { return (unsigned)((((int64_t)slots * kv_heads + 7) / 8) * 8 * group); }

// ends[s - 1], held to 0 .. T: whatever the array holds, no row outside the caller's is touched
__device__ __forceinline__ int packed_end(const PackedAttention& p, int s) { return s > 0 ? min(max(p.ends[s - 1], 0), p.T) : 0; }

// the sequence of a slot: the last s with f(s) <= slot, in steps of 64 (one load for up to 64 sequences)
template <int M>
__device__ __forceinline__ bool packed_rows(const PackedAttention& p, int slot, PackedPlace& w) {
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

// A block of one query head; false: it has no rows.  A sequence's last rows come first: with a causal mask they have most work.
template <int M>
__device__ __forceinline__ bool packed_place(const PackedAttention& p, int slots, PackedPlace& w) {
  const int group = p.n_heads / p.n_kv_heads, i = blockIdx.x >> 3;
  const int unit = i / group * 8 + (blockIdx.x & 7), slot = unit / p.n_kv_heads;
  if (slot >= slots) return false;
  w.kv = __builtin_amdgcn_readfirstlane(unit - slot * p.n_kv_heads);
  w.head = __builtin_amdgcn_readfirstlane(w.kv * group + i % group);
  return packed_rows<M>(p, slots - 1 - slot, w);
}
// A block of all query heads of one head of keys; first_first: a sequence's first rows come first.
template <int M>
__device__ __forceinline__ bool packed_place_kv(const PackedAttention& p, int slots, bool first_first, PackedPlace& w) {
  const int slot = (int)blockIdx.x / p.n_kv_heads;
  if (slot >= slots) return false;
  w.kv = __builtin_amdgcn_readfirstlane((int)blockIdx.x - slot * p.n_kv_heads);
  w.head = w.kv * (p.n_heads / p.n_kv_heads);
  return packed_rows<M>(p, first_first ? slot : slots - 1 - slot, w);
}

}  // namespace mk
