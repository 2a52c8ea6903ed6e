// Attention of a drafted tree over the retained cache: how the cache rows are dealt to CTAs, the tiles
// of a slice, and the layout of the partial results.
#pragma once
#include "common.cuh"
#include "decode_common.cuh"

namespace tca {

// Rows of a unit's query block: row r = head-of-group * T + drafted token, as they lie in q.
struct TreePlan {
  int rows;          // G * T
  int rows_per_cta;
  int row_blocks;    // CTAs per slice
  int streams;       // partial results a CTA writes per row
  int n_slots;       // slices of all units together, at most
  int step_rows;     // slices are multiples of this many rows ...
  int min_steps;     // ... and at least this many steps long
};
TreePlan tree_plan(const tca_params* prm, int n_draft);

// Workspace: 256-byte header (word 0: sticky status), one (first slot, slices) pair per unit, the row
// statistics (maximum in log2 units, sum) and the unnormalised outputs of every (slot, stream, row).
constexpr size_t kTreeHeaderBytes = 256;
struct TreeWs {
  int* status;
  int2* table;      // [units]
  float2* ml;       // [n_slots * streams][rows]
  float* acc;       // [n_slots * streams][rows][d]
  size_t bytes;
};
inline TreeWs tree_ws_layout(const tca_params* prm, const TreePlan& p, void* ws) {
  TreeWs w;
  const size_t U = size_t(prm->batch) * prm->n_kv_heads, n = size_t(p.n_slots) * p.streams * p.rows;
  char* base = static_cast<char*>(ws);
  size_t at = kTreeHeaderBytes;
  w.status = reinterpret_cast<int*>(base);
  w.table = reinterpret_cast<int2*>(base + at);
  at += align_up(U * sizeof(int2), 256);
  w.ml = reinterpret_cast<float2*>(base + at);
  at += align_up(n * sizeof(float2), 256);
  w.acc = reinterpret_cast<float*>(base + at);
  w.bytes = at + align_up(n * prm->head_dim * sizeof(float), 256);
  return w;
}

// The rows of one slice: up to three runs of physically contiguous cache rows (global region, ring up
// to its end, ring from its start), walked in tiles of `tile` rows; the last tile of a run may be short.
struct SliceTiles {
  int y[3], n[3];
  int tile;
  __device__ __forceinline__ int count(int i) const { return (n[i] + tile - 1) / tile; }
  __device__ __forceinline__ int n_tiles() const { return count(0) + count(1) + count(2); }
  // first cache row of tile t and the rows it holds
  __device__ __forceinline__ void get(int t, int& row, int& rows) const {
    int i = 0;
    if (t >= count(0)) {
      t -= count(0);
      i = 1;
      if (t >= count(1)) {
        t -= count(1);
        i = 2;
      }
    }
    const int yi = i == 0 ? y[0] : i == 1 ? y[1] : y[2], ni = i == 0 ? n[0] : i == 1 ? n[1] : n[2];
    row = yi + t * tile;
    rows = min(tile, ni - t * tile);
  }
};

// A slice of a unit's rows.
struct TreeSlice {
  int u;             // -1: no such slice
  int part, np;      // slice within the unit, slices of the unit
  int base;          // slot of the unit's first slice
  SliceTiles tiles;
};

// The lin-th slice over all units.  Rows are dealt in steps of `step` rows; the slice length is the
// smallest multiple of it for which no more than n_slots slices exist, so the slices of all units fit the
// launch whatever the cache holds.  It is worked out from the device's state words: a captured launch
// stays right when the cache has grown since.  Whole warp; every lane returns the same.
__device__ __forceinline__ TreeSlice tree_find(const int64_t* state, int n_units, int64_t tail_cap, int n_slots, int step,
                                               int min_steps, int tile, int lin, int lane) {
  constexpr int kHeld = 4;   // units held in registers per lane; more are read again
  const int groups = min(kHeld, (n_units + 31) / 32);
  auto steps_of = [&](int u) -> int {
    if (u >= n_units) return 0;
    const int64_t* st = state + size_t(u) * TCA_STATE_WORDS;
    return int((st[TCA_ST_N_GLOBAL] + st[TCA_ST_N_TAIL] + step - 1) / step);
  };
  int held[kHeld], most = 0, sum = 0;
  UnitView first{};          // the view of unit `lane`, for the units most calls have
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    held[k] = 0;
    if (k >= groups) continue;
    if (k == 0) {
      if (lane < n_units) first = load_unit(state, lane, tail_cap);
      held[0] = int((first.len() + step - 1) / step);
    } else {
      held[k] = steps_of(k * 32 + lane);
    }
    most = max(most, held[k]);
    sum += held[k];
  }
  for (int u = 32 * kHeld + lane; u < n_units; u += 32) {
    const int n = steps_of(u);
    most = max(most, n);
    sum += n;
  }
  most = __reduce_max_sync(0xffffffffu, most);
  sum = __reduce_add_sync(0xffffffffu, sum);
  auto count = [&](int per) {   // slices of at most `per` steps
    int c = 0;
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (k < groups) c += (held[k] + per - 1) / per;
    for (int u = 32 * kHeld + lane; u < n_units; u += 32) c += (steps_of(u) + per - 1) / per;
    return int(__reduce_add_sync(0xffffffffu, c));
  };
  // count(per) <= sum / per + n_units, which bounds the search from above
  int lo = max(min_steps, (sum + n_slots - 1) / n_slots);
  int hi = max(lo, n_slots > n_units ? min(most, (sum + n_slots - n_units - 1) / (n_slots - n_units)) : most);
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (count(mid) <= n_slots) hi = mid; else lo = mid + 1;
  }
  TreeSlice s;
  s.u = -1;
  int offset = 0;
  for (int k = 0; k * 32 < n_units; ++k) {
    int mine = 0;
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
      if (h == k) mine = held[h];
    if (k >= kHeld) mine = steps_of(k * 32 + lane);
    const int np = (mine + lo - 1) / lo;
    int incl = np;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, incl, off);
      if (lane >= off) incl += t;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, lin < offset + incl);
    if (hit) {
      const int l = __ffs(hit) - 1;
      s.u = k * 32 + l;
      s.np = __shfl_sync(0xffffffffu, np, l);
      s.base = offset + __shfl_sync(0xffffffffu, incl - np, l);
      s.part = lin - s.base;
      break;
    }
    offset += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (s.u < 0) return s;
  UnitView v;
  if (s.u < 32) {
    v.seg = __shfl_sync(0xffffffffu, first.seg, s.u);
    v.gcap = __shfl_sync(0xffffffffu, first.gcap, s.u);
    v.n_global = __shfl_sync(0xffffffffu, first.n_global, s.u);
    v.tail_head = __shfl_sync(0xffffffffu, first.tail_head, s.u);
    v.n_tail = __shfl_sync(0xffffffffu, first.n_tail, s.u);
    v.tail_cap = tail_cap;
  } else {
    v = load_unit(state, s.u, tail_cap);
  }
  const int64_t len = v.len(), n_steps = (len + step - 1) / step;
  const int64_t r0 = slice_begin(n_steps, s.np, s.part) * step;
  const int64_t r1 = min(len, slice_begin(n_steps, s.np, s.part + 1) * step);
  s.tiles.tile = tile;
  int64_t r = r0;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int64_t n = r < r1 ? (r < v.n_global ? min(r1, v.n_global) - r : v.run(r, r1 - r)) : 0;
    s.tiles.y[i] = n > 0 ? int(v.phys(r)) : 0;
    s.tiles.n[i] = int(n);
    r += n;
    // a slice that begins inside the ring has no first run in the global region: the order is the same
  }
  return s;
}

}  // namespace tca
