// Attention of a drafted tree over the retained cache: how the cache rows are dealt to CTAs, the tiles
// of a slice, and the layout of the partial results.
#pragma once
#include "common.cuh"

namespace tca {

// Rows of a unit's query block: row r = head-of-group * T + drafted token, as they lie in q.
struct TreePlan {
  int rows;          // G * T
  int rows_per_cta;
  int row_blocks;    // CTAs per share of the cache rows, one per rows_per_cta query rows
  int streams;       // partial results a CTA writes per row
  int min_share;     // steps of kTreeStep rows: a shorter share is all latency
  int lead;          // steps that starting on a unit costs
  int n_shares;      // shares the cache rows of all units are cut into, at most
  int n_slots;       // slots for partial results: a share touches a run of units, so (share, unit) pairs
                     // number at most n_shares + units
};
TreePlan tree_plan(const tca_params* prm, int n_draft);

// Workspace: 256-byte header (word 0: sticky status), one (first slot, slots) pair per unit, the row
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

// The rows of one piece of a unit: up to three runs of physically contiguous cache rows (global region,
// ring up to its end, ring from its start), in tiles of kTile rows: first the full tiles of all runs, then
// what is left of each run that is not a multiple of it.  (The order does not matter to the attention.)
template <int kTile>
struct SliceTiles {
  int y[3], n[3];
  __device__ __forceinline__ int full(int i) const { return int(unsigned(n[i]) / unsigned(kTile)); }
  __device__ __forceinline__ int n_whole() const { return full(0) + full(1) + full(2); }
  __device__ __forceinline__ int n_tiles() const {
    return n_whole() + (n[0] % kTile != 0) + (n[1] % kTile != 0) + (n[2] % kTile != 0);
  }
  // first cache row of tile t and the rows it holds
  __device__ __forceinline__ void get(int t, int& row, int& rows) const {
    const int f0 = full(0), f1 = full(1), f2 = full(2);
    rows = kTile;
    if (t < f0) { row = y[0] + t * kTile; return; }
    t -= f0;
    if (t < f1) { row = y[1] + t * kTile; return; }
    t -= f1;
    if (t < f2) { row = y[2] + t * kTile; return; }
    t -= f2;
    const int r0 = n[0] - f0 * kTile, r1 = n[1] - f1 * kTile, r2 = n[2] - f2 * kTile;
    if (r0 > 0 && t-- == 0) { row = y[0] + f0 * kTile; rows = r0; return; }
    if (r1 > 0 && t-- == 0) { row = y[1] + f1 * kTile; rows = r1; return; }
    row = y[2] + f2 * kTile;
    rows = r2;
  }
};

// What one CTA attends to at a time: a piece of a unit's rows.
template <int kTile>
struct TreePiece {
  int u;
  int slot;          // where its partial results go
  SliceTiles<kTile> tiles;
};

// How the cache rows of all units are dealt: laid end to end in steps of kTreeStep rows, they are cut into
// equal shares, one per CTA (per block of query rows), wherever the cuts fall; a share that runs into
// the next unit works on both, one after the other.  A unit counts plan.lead steps more than it has, because
// starting on one costs about that much.  (Giving each unit a whole number of slices of its own left the
// longest 13 % above the mean with 32 units of 65 to 142 steps.)  The pair (share i, unit u) has slot i + u:
// pairs advance in one of the two at a time, so slots are distinct and a unit's are consecutive.
// The cuts follow from the device's state words, not from the host's mirror: a captured launch stays right
// when the cache has grown since.  Whole warp; every lane returns the same.  All 32-bit (a cache has
// fewer than 2^31 rows), no 64-bit divisions: this stands between the launch and the first load.
constexpr int kTreeStep = 128, kTreeStepLog = 7;

struct TreeFinder {
  int lead;
  int q, longer;      // shares are q steps, the first `longer` of them q + 1
  int begin, end;     // this CTA's share
  int u0, offset;     // group of 32 units the walk is at, steps before it
  unsigned done;      // units of the group that were handed out

  __device__ __forceinline__ static int steps_of(const int64_t* state, int n_units, int u) {
    if (u >= n_units) return 0;
    const int64_t* st = state + size_t(u) * TCA_STATE_WORDS;
    return int((st[TCA_ST_N_GLOBAL] + st[TCA_ST_N_TAIL] + kTreeStep - 1) >> kTreeStepLog);
  }
  __device__ __forceinline__ int share_of(int x) const {   // the share that holds step x
    const int head = longer * (q + 1);
    return x < head ? x / (q + 1) : longer + (x - head) / q;
  }
  __device__ __forceinline__ void start(const int64_t* state, int n_units, const TreePlan& plan, int share, int lane) {
    lead = plan.lead;
    int total = 0;
    for (int u = lane; u < n_units; u += 32) {
      const int n = steps_of(state, n_units, u);
      total += n > 0 ? n + lead : 0;
    }
    total = __reduce_add_sync(0xffffffffu, total);
    const int n = max(1, min(plan.n_shares, int(unsigned(total) / unsigned(plan.min_share))));
    q = int(unsigned(total) / unsigned(n));
    longer = total - q * n;
    begin = share < n ? share * q + min(share, longer) : total;
    end = share < n ? begin + q + (share < longer ? 1 : 0) : total;
    u0 = offset = 0;
    done = 0;
  }
  // The next piece of this share; false after the last.  The first piece of a unit also records where the
  // unit's partial results lie.
  template <int kTile>
  __device__ __forceinline__ bool next(const int64_t* state, int n_units, int tail_cap, int share, bool record, int2* table,
                                       int lane, TreePiece<kTile>& p) {
    for (; u0 < n_units && offset < end; u0 += 32, done = 0) {
      const int steps = steps_of(state, n_units, u0 + lane);
      const int width = steps > 0 ? steps + lead : 0;
      int incl = width;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += t;
      }
      const int at = offset + incl - steps;              // where the unit's rows begin
      const int lo = max(at, begin), hi = min(at + steps, end);
      const unsigned hit = __ballot_sync(0xffffffffu, hi > lo) & ~done;
      if (hit == 0) {
        offset += __shfl_sync(0xffffffffu, incl, 31);
        continue;
      }
      const int l = __ffs(hit) - 1;
      done |= 1u << l;
      p.u = u0 + l;
      p.slot = share + p.u;
      const int at_l = __shfl_sync(0xffffffffu, at, l), steps_l = __shfl_sync(0xffffffffu, steps, l);
      const int s0 = __shfl_sync(0xffffffffu, lo, l) - at_l, s1 = __shfl_sync(0xffffffffu, hi, l) - at_l;
      if (s0 == 0 && record && lane == 0)
        table[p.u] = make_int2(p.slot, share_of(at_l + steps_l - 1) - share + 1);
      const int64_t* st = state + size_t(p.u) * TCA_STATE_WORDS;
      const int seg = int(st[TCA_ST_SEG_START]), gcap = int(st[TCA_ST_GLOBAL_CAP]), ng = int(st[TCA_ST_N_GLOBAL]);
      const int head = int(st[TCA_ST_TAIL_HEAD]), len = ng + int(st[TCA_ST_N_TAIL]);
      const int r0 = s0 * kTreeStep, r1 = min(len, s1 * kTreeStep);
      // runs: rows [r0, r1) of the global region, then of the ring up to its end, then from its start
      const int wrap = ng + tail_cap - head;             // logical row that lies in the ring's slot 0
      const int b1 = min(max(ng, r0), r1), b2 = max(min(max(wrap, r0), r1), b1);
      p.tiles.y[0] = seg + r0;
      p.tiles.n[0] = b1 - r0;
      p.tiles.y[1] = seg + gcap + head + (b1 - ng);
      p.tiles.n[1] = b2 - b1;
      p.tiles.y[2] = seg + gcap + (b2 - wrap);
      p.tiles.n[2] = r1 - b2;
      return true;
    }
    return false;
  }
};

}  // namespace tca
