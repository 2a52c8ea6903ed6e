// Packed prompts: the view of the caller's strided buffers and the search that tells a CTA which
// query positions of which sequence it works on.
#pragma once
#include "common.cuh"

namespace tca {

// Element strides of one packed buffer [heads, rows, head_dim].
struct PackedView {
  int64_t head, row;
};
struct PackedArgs {
  PackedView q, k, v, o;
  int64_t rows;                 // rows of every buffer
  const int64_t* seq_start;     // DEVICE [n_seq + 1]
  int n_seq, n_q_heads, n_kv_heads;
};

// What one CTA does: query positions [p0, p0 + n_pos) of the sequence that begins at row `row0` and
// is `len` tokens long, for the query heads of one KV head.
struct PackedWork {
  int64_t row0;
  int len, p0, kvh;
};

// Work items are (sequence, tile of `tile_pos` positions), per KV head.  Their number follows from the
// device offsets, which the host does not read: it launches packed_max_tiles() CTAs per KV head, an
// upper bound for disjoint sequences, and the CTAs past the end leave at once.  Offsets that are not
// ascending or leave [0, rows] are clamped, so no CTA ever addresses a row outside the buffers.
inline int64_t packed_max_tiles(int64_t rows, int n_seq, int tile_pos) { return rows / tile_pos + n_seq; }

__device__ __forceinline__ void packed_bounds(const PackedArgs& a, int s, int64_t& lo, int& len) {
  lo = min(max(a.seq_start[s], int64_t(0)), a.rows);
  const int64_t hi = min(max(a.seq_start[s + 1], int64_t(0)), a.rows);
  len = hi > lo ? int(hi - lo) : 0;
}

// The i-th work item, longest first (a causal tile costs its index): among all tiles, in descending
// order of their index within their sequence, then by ascending sequence.  With C(j) = sum over the
// sequences of max(0, tiles - j), tile index j holds items [C(j+1), C(j)): a binary search over j, no
// list in memory.  Whole warp; every lane returns the same.  False: there is no i-th item.
// Up to 128 sequences are held in registers (four per lane), more are read again per probe.
__device__ __forceinline__ bool packed_find(const PackedArgs& a, int64_t i, int tile_pos, int lane, int& seq, int& tile) {
  constexpr int kHeld = 4;
  int held[kHeld];
  const bool in_regs = a.n_seq <= 32 * kHeld;
  auto tiles_of = [&](int s) -> int {
    if (s >= a.n_seq) return 0;
    int64_t lo;
    int len;
    packed_bounds(a, s, lo, len);
    return (len + tile_pos - 1) / tile_pos;
  };
  int mx = 0;
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    held[k] = tiles_of(k * 32 + lane);
    mx = max(mx, held[k]);
  }
  for (int s = 32 * kHeld + lane; s < a.n_seq; s += 32) mx = max(mx, tiles_of(s));
  mx = __reduce_max_sync(0xffffffffu, mx);
  auto count_from = [&](int j) -> int64_t {   // C(j); fits 32 bits because rows do
    int c = 0;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) c += max(0, held[k] - j);
    if (!in_regs)
      for (int s = 32 * kHeld + lane; s < a.n_seq; s += 32) c += max(0, tiles_of(s) - j);
    return int64_t(__reduce_add_sync(0xffffffffu, c));
  };
  int lo = 0, hi = mx;             // the largest j with C(j) > i; C(mx) = 0
  if (mx == 0 || count_from(0) <= i) return false;
  while (hi - lo > 1) {            // C(lo) > i >= C(hi)
    const int mid = (lo + hi) >> 1;
    if (count_from(mid) > i) lo = mid; else hi = mid;
  }
  int rank = int(i - count_from(lo + 1));   // among the sequences with more than lo tiles
  tile = lo;
  for (int k = 0; k * 32 < a.n_seq; ++k) {
    int n = 0;
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
      if (h == k) n = held[h];
    if (k >= kHeld) n = tiles_of(k * 32 + lane);
    unsigned m = __ballot_sync(0xffffffffu, n > lo);
    const int c = __popc(m);
    if (rank < c) {
      seq = k * 32 + int(__fns(m, 0, rank + 1));
      return true;
    }
    rank -= c;
  }
  return false;   // only if the offsets overlap
}

}  // namespace tca
