// Attention of a drafted tree over the retained cache: how the cache rows are dealt to CTAs, the tiles
// of a slice, and the layout of the partial results.
#pragma once
#include "common.cuh"

namespace tca {

// Rows of a unit's query block: row r = head-of-group * T + drafted token, as they lie in q.
struct TreePlan {
  int rows;          // G * T
  int rows_per_cta;
  int row_blocks;    // CTAs per slice
  int streams;       // partial results a CTA writes per row
  int n_slots;       // slices of all units together, at most
  int min_steps;     // shortest slice, in steps of kTreeStep rows
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

// The lin-th slice over all units.  Rows are dealt in steps of kTreeStep rows; the slice length is the
// smallest multiple of it for which no more than n_slots slices exist, so the slices of all units fit the
// launch whatever the cache holds.  It is worked out from the device's state words: a captured launch
// stays right when the cache has grown since.  Whole warp; every lane returns the same.  Everything is
// 32-bit (a cache has fewer than 2^31 rows) and without 64-bit divisions: this stands between the launch and
// the first load (3700 -> 1500 clocks).
constexpr int kTreeStep = 128, kTreeStepLog = 7;

__device__ __forceinline__ TreeSlice tree_find(const int64_t* state, int n_units, int tail_cap, int n_slots, int min_steps,
                                               int tile, int lin, int lane) {
  int n_global = 0, n_tail = 0;     // unit `lane`; units past the 32nd are read again in every pass
  if (lane < n_units) {
    const int64_t* st = state + size_t(lane) * TCA_STATE_WORDS;
    n_global = int(st[TCA_ST_N_GLOBAL]);
    n_tail = int(st[TCA_ST_N_TAIL]);
  }
  const int first = (n_global + n_tail + kTreeStep - 1) >> kTreeStepLog;
  auto steps_of = [&](int u) -> int {
    if (u >= n_units) return 0;
    const int64_t* st = state + size_t(u) * TCA_STATE_WORDS;
    return int((st[TCA_ST_N_GLOBAL] + st[TCA_ST_N_TAIL] + kTreeStep - 1) >> kTreeStepLog);
  };
  int most = first, sum = first;
  for (int u = 32 + lane; u < n_units; u += 32) {
    const int n = steps_of(u);
    most = max(most, n);
    sum += n;
  }
  most = __reduce_max_sync(0xffffffffu, most);
  sum = __reduce_add_sync(0xffffffffu, sum);
  auto parts = [](int steps, int per) { return int((unsigned(steps) + unsigned(per) - 1u) / unsigned(per)); };
  // slices of `per` steps number at most sum / per + n_units, which bounds the search from above
  int lo = max(min_steps, parts(sum, n_slots));
  int hi = max(lo, n_slots > n_units ? min(most, parts(sum, n_slots - n_units)) : most);
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    int c = parts(first, mid);
    for (int u = 32 + lane; u < n_units; u += 32) c += parts(steps_of(u), mid);
    if (int(__reduce_add_sync(0xffffffffu, c)) <= n_slots) hi = mid; else lo = mid + 1;
  }
  TreeSlice s;
  s.u = -1;
  int offset = 0, steps = 0;
  for (int u0 = 0; u0 < n_units; u0 += 32) {
    const int mine = u0 == 0 ? first : steps_of(u0 + lane);
    const int np = parts(mine, lo);
    int incl = np;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, incl, off);
      if (lane >= off) incl += t;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, lin < offset + incl);
    if (hit) {
      const int l = __ffs(hit) - 1;
      s.u = u0 + l;
      s.np = __shfl_sync(0xffffffffu, np, l);
      s.base = offset + __shfl_sync(0xffffffffu, incl - np, l);
      steps = __shfl_sync(0xffffffffu, mine, l);
      s.part = lin - s.base;
      break;
    }
    offset += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (s.u < 0) return s;
  const int64_t* st = state + size_t(s.u) * TCA_STATE_WORDS;
  const int seg = int(st[TCA_ST_SEG_START]), gcap = int(st[TCA_ST_GLOBAL_CAP]), ng = int(st[TCA_ST_N_GLOBAL]);
  const int head = int(st[TCA_ST_TAIL_HEAD]), len = ng + int(st[TCA_ST_N_TAIL]);
  // the unit's steps dealt evenly: the first `longer` slices have one more
  const int each = int(unsigned(steps) / unsigned(s.np)), longer = steps - each * s.np;
  const int r0 = (s.part * each + min(s.part, longer)) * kTreeStep;
  const int r1 = min(len, r0 + (each + (s.part < longer ? 1 : 0)) * kTreeStep);
  // runs: rows [r0, r1) of the global region, then of the ring up to its end, then from its start
  const int wrap = ng + tail_cap - head;      // logical row that lies in the ring's slot 0
  const int b1 = min(max(ng, r0), r1), b2 = min(max(wrap, r0), r1);
  s.tiles.tile = tile;
  s.tiles.y[0] = seg + r0;
  s.tiles.n[0] = b1 - r0;
  s.tiles.y[1] = seg + gcap + head + (b1 - ng);
  s.tiles.n[1] = max(b2, b1) - b1;
  s.tiles.y[2] = seg + gcap + (max(b2, b1) - wrap);
  s.tiles.n[2] = r1 - max(b2, b1);
  return s;
}

}  // namespace tca
