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
// list in memory.  A whole warp works on it; up to 128 sequences are read once and held in registers
// (four per lane, the loads and the search are then a few hundred clocks), more are read again per probe.
struct PackedFinder {
  static constexpr int kHeld = 4;
  int tiles[kHeld], row0[kHeld], len[kHeld];

  __device__ __forceinline__ static int tiles_of(const PackedArgs& a, int s, int tile_pos) {
    if (s >= a.n_seq) return 0;
    int64_t lo;
    int n;
    packed_bounds(a, s, lo, n);
    return (n + tile_pos - 1) / tile_pos;
  }
  __device__ __forceinline__ void read(const PackedArgs& a, int tile_pos, int lane) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      tiles[k] = row0[k] = len[k] = 0;
      if (k * 32 + lane < a.n_seq) {
        int64_t lo;
        packed_bounds(a, k * 32 + lane, lo, len[k]);
        row0[k] = int(lo);
        tiles[k] = (len[k] + tile_pos - 1) / tile_pos;
      }
    }
  }
  // Every lane returns the same.  False: there is no i-th item.
  __device__ __forceinline__ bool find(const PackedArgs& a, int i, int tile_pos, int lane, int64_t& row, int& n, int& tile) const {
    const int held = min(kHeld, (a.n_seq + 31) / 32);
    int mx = 0;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) mx = max(mx, tiles[k]);
    for (int s = 32 * kHeld + lane; s < a.n_seq; s += 32) mx = max(mx, tiles_of(a, s, tile_pos));
    mx = __reduce_max_sync(0xffffffffu, mx);
    auto count_from = [&](int j) {   // C(j); fits 32 bits because rows do
      int c = max(0, tiles[0] - j);
#pragma unroll
      for (int k = 1; k < kHeld; ++k)
        if (k < held) c += max(0, tiles[k] - j);
      for (int s = 32 * kHeld + lane; s < a.n_seq; s += 32) c += max(0, tiles_of(a, s, tile_pos) - j);
      return __reduce_add_sync(0xffffffffu, c);
    };
    int lo = 0, hi = mx, above = 0;  // the largest j with C(j) > i; C(mx) = 0
    if (mx == 0 || count_from(0) <= i) return false;
    while (hi - lo > 1) {            // C(lo) > i >= C(hi) = above
      const int mid = (lo + hi) >> 1, c = count_from(mid);
      if (c > i) lo = mid; else { hi = mid; above = c; }
    }
    int rank = i - above;            // among the sequences with more than lo tiles
    tile = lo;
    for (int k = 0; k * 32 < a.n_seq; ++k) {
      int mine = 0, r0 = 0, ln = 0;
#pragma unroll
      for (int h = 0; h < kHeld; ++h)
        if (h == k) { mine = tiles[h]; r0 = row0[h]; ln = len[h]; }
      if (k >= kHeld) mine = tiles_of(a, k * 32 + lane, tile_pos);
      const unsigned m = __ballot_sync(0xffffffffu, mine > lo);
      const int c = __popc(m);
      if (rank < c) {
        const unsigned hit = __ballot_sync(0xffffffffu, mine > lo && __popc(m & ((1u << lane) - 1u)) == rank);
        const int l = __ffs(hit) - 1;
        if (k < kHeld) {
          row = __shfl_sync(0xffffffffu, r0, l);
          n = __shfl_sync(0xffffffffu, ln, l);
        } else {
          packed_bounds(a, k * 32 + l, row, n);
        }
        return true;
      }
      rank -= c;
    }
    return false;   // only if the offsets overlap
  }
};

}  // namespace tca
