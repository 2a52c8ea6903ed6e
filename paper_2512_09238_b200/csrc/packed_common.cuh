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

// Finds the i-th work item.  A whole warp works on it.
//
// Up to 128 sequences: longest first (a causal tile costs its index), that is among all tiles in descending
// order of their index within their sequence, then by ascending sequence.  With C(j) = sum over the
// sequences of max(0, tiles - j), tile index j holds items [C(j+1), C(j)): a binary search over j, no list
// in memory, the tile counts in shared memory.
// More sequences: in their own order, the longest tile of each first, found by walking on from the last item
// (a CTA asks for ascending i).  The search above would read all of them several times per item (2000 short
// prompts: 10.8 ms against 1.6 ms).  The order matters little if they are short; one prompt of 16K tokens among 127
// of 100 takes 1.96 ms, among 128 of them 1.99 ms, one of 128K among those of 20 116 and 119 to 120 ms (that
// includes the order of the heads, see launch_packed_tc).
//
// Loops are left rolled: the search runs beside the arithmetic of the item before, and code that is not
// there does not push that out of the instruction cache.
struct PackedFinder {
  static constexpr int kHeld = 128;
  int* held;      // shared memory [kHeld]
  int most;       // sorted: no sequence has more tiles.  Walk: -1
  int s0, offset; // walk: first sequence of the group of 32 it is at, items before that

  __device__ __forceinline__ static int tiles_of(const PackedArgs& a, int s, int tile_pos) {
    int64_t lo;
    int n;
    packed_bounds(a, s, lo, n);
    return int(unsigned(n + tile_pos - 1) / unsigned(tile_pos));
  }
  __device__ __forceinline__ void read(const PackedArgs& a, int tile_pos, int lane, int* shared) {
    held = shared;
    most = -1;
    s0 = offset = 0;
    if (a.n_seq > kHeld) return;
    int mx = 0;
#pragma unroll 1
    for (int s = lane; s < a.n_seq; s += 32) {
      held[s] = tiles_of(a, s, tile_pos);
      mx = max(mx, held[s]);
    }
    most = __reduce_max_sync(0xffffffffu, mx);
    __syncwarp();
  }
  // Every lane returns the same.  False: there is no i-th item.
  __device__ __forceinline__ bool find(const PackedArgs& a, int i, int tile_pos, int lane, int64_t& row, int& n, int& tile) {
    if (most < 0) {
      if (i < offset) s0 = offset = 0;     // the next head begins anew
#pragma unroll 1
      for (; s0 < a.n_seq; s0 += 32) {
        const int mine = s0 + lane < a.n_seq ? tiles_of(a, s0 + lane, tile_pos) : 0;
        int incl = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const int t = __shfl_up_sync(0xffffffffu, incl, off);
          if (lane >= off) incl += t;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, i < offset + incl);
        if (hit) {
          const int l = __ffs(hit) - 1;
          tile = __shfl_sync(0xffffffffu, offset + incl, l) - 1 - i;
          packed_bounds(a, s0 + l, row, n);
          return true;
        }
        offset += __shfl_sync(0xffffffffu, incl, 31);
      }
      return false;
    }
    int lo = -1, hi = most, above = 0;     // the largest j with C(j) > i; C(most) = 0 = above
#pragma unroll 1
    while (hi - lo > 1) {                  // C(lo) > i >= C(hi)
      const int mid = (lo + hi) >> 1;
      int c = 0;                           // fits 32 bits because rows do
#pragma unroll 1
      for (int s = lane; s < a.n_seq; s += 32) c += max(0, held[s] - mid);
      c = __reduce_add_sync(0xffffffffu, c);
      if (c > i) lo = mid; else { hi = mid; above = c; }
    }
    if (lo < 0) return false;
    int rank = i - above;                  // among the sequences with more than lo tiles
    tile = lo;
#pragma unroll 1
    for (int g = 0; g < a.n_seq; g += 32) {
      const bool in = g + lane < a.n_seq && held[g + lane] > lo;
      const unsigned m = __ballot_sync(0xffffffffu, in);
      const unsigned hit = __ballot_sync(0xffffffffu, in && __popc(m & ((1u << lane) - 1u)) == rank);
      if (hit) {
        packed_bounds(a, g + __ffs(hit) - 1, row, n);
        return true;
      }
      rank -= __popc(m);
    }
    return false;   // only if the offsets overlap
  }
};

}  // namespace tca
