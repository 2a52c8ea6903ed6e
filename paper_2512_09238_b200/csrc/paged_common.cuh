// The paged cache: which slots a new token sees, how the visible rows of all units are dealt to CTAs, and the layout of
// the partial results of tca_attn_paged.
#pragma once
#include "common.cuh"
#include "ptx_sm100.cuh"

namespace tca {

enum { kPagedNoRoom = 1, kPagedBadPage = 2, kPagedBudget = 3 };   // state word TCA_PG_CHECK

int check_paged(const tca_params* prm, const tca_paged_desc* c);   // paged.cu

// What kernels need of the descriptor.
struct PagedArgs {
  const int32_t* table;    // [units][max_pages]
  int4* state;             // [units]
  int n_units, max_pages, page_shift;
  int n_pages;
};
inline PagedArgs paged_args(const tca_paged_desc* c) {
  PagedArgs a;
  a.table = c->table;
  a.state = reinterpret_cast<int4*>(c->state);
  a.n_units = int(c->n_units);
  a.max_pages = c->max_pages;
  a.page_shift = 0;
  while ((1 << a.page_shift) < c->page_size) ++a.page_shift;
  a.n_pages = int(c->n_pages);
  return a;
}

#ifdef __CUDACC__
__device__ __forceinline__ int paged_len(const PagedArgs& a, int len) { return min(max(len, 0), a.max_pages << a.page_shift); }
// Pool row of a unit's slot; -1: the table holds no page of the pool there.
__device__ __forceinline__ int paged_row(const PagedArgs& a, int u, int slot) {
  const int page = a.table[size_t(u) * a.max_pages + (slot >> a.page_shift)];
  return unsigned(page) < unsigned(a.n_pages) ? (page << a.page_shift) + (slot & ((1 << a.page_shift) - 1)) : -1;
}
__device__ __forceinline__ void report_paged(int4* unit_state, int which) {
  atomicCAS(reinterpret_cast<int*>(unit_state) + TCA_PG_CHECK, 0, which);
}
#endif

// The slots of a unit in steps of 128: first those that hold sinks, then those from the first slot of the window on
// (a step that holds both counts once).
constexpr int kPagedStep = 128;
struct PagedSpan {
  int len, sinks, lo;      // visible: slot < len and (slot < sinks or slot >= lo)
  int n0, first, n;        // steps that hold sinks, step the others begin with, steps in all
#ifdef __CUDACC__
  __device__ __forceinline__ PagedSpan(int length, int window, int n_sink) {
    len = length;
    lo = max(0, len - window);
    sinks = min(n_sink, lo);
    n0 = (sinks + kPagedStep - 1) / kPagedStep;
    first = max(n0, lo / kPagedStep);
    n = n0 + max(0, (len + kPagedStep - 1) / kPagedStep - first);
  }
  __device__ __forceinline__ int slot0(int step) const { return (step < n0 ? step : first + step - n0) * kPagedStep; }
  // bit i: slot0 + i is visible (16 slots)
  __device__ __forceinline__ unsigned visible16(int slot) const {
    auto below = [&](int n) { return n >= 16 ? 0xffffu : n <= 0 ? 0u : (1u << n) - 1u; };
    return below(len - slot) & (below(sinks - slot) | ~below(lo - slot));
  }
  __device__ __forceinline__ bool any_visible(int slot, int n) const {
    return slot < sinks || (slot + n > lo && slot < len);
  }
#endif
};

// How the steps of all units are dealt: laid end to end they are cut into equal shares, one per CTA, wherever the cuts
// fall; a share that runs into the next unit works on both.  The cuts follow from the device's state, so a captured launch
// stays right when the cache has changed since.  Pair (share i, unit u) has partial slot i + u: pairs advance in one of
// the two at a time, so slots are distinct and a unit's are consecutive.  A unit is kPagedLead wider than its steps are,
// which is what starting on one and finishing it costs.
// (The SMs do not get the same bandwidth: of 249 MB the first finish after 42 us, half of them after 45, the last after 51.
// A quarter of the steps in small shares that whoever is ready takes did not help: what a CTA has to ask for ahead, three
// small shares, takes as long as that, and finding them delayed the start: 76 against 58 us.)
constexpr int kPagedLead = 1;
struct PagedCut {
  int total, n, q, longer;               // width; shares: the first `longer` are q + 1 wide, the others q
#ifdef __CUDACC__
  __host__ __device__ PagedCut(int steps, int ctas) {
    total = steps;
    n = steps < ctas ? (steps > 0 ? steps : 1) : ctas;
    q = int(unsigned(steps) / unsigned(n));
    longer = steps - q * n;
  }
  __device__ __forceinline__ int begin(int share) const { return share < n ? share * q + min(share, longer) : total; }
  __device__ __forceinline__ int share_of(int x) const {   // the share that place x lies in
    const int head = longer * (q + 1);
    return x < head ? int(unsigned(x) / unsigned(q + 1)) : longer + int(unsigned(x - head) / unsigned(q));
  }
#endif
};
struct PagedPiece {
  int u, s0, n;            // steps [s0, s0 + n) of unit u
  int len;                 // rows of the unit
  int step;                // steps of the units before it
  int slot, parts;         // the unit's partial results: first slot, number (0: this piece is all it has)
};
// What the second kernel needs of a share, and of a step.
struct __align__(16) PagedRecord {
  int u, slot, parts;      // the unit that runs from the share into the next, its partial results; parts 0: there is none
  int steps;               // of all units
};
struct __align__(16) PagedStepRecord {
  int2 group[8];           // of every 16 slots: pool row / 16 (-1: not a page of the pool), visible slots as bits
  int slot, parts, unused[2];
};

#ifdef __CUDACC__
// The CTA's first kDealers threads lay the steps end to end: one trip to memory for all rows (kept meanwhile in shared
// memory that the caller needs only later; copied_over: for bulk copies), a thread takes a run of units, a scan of their widths.  All threads take part in the barriers.  The share's
// pieces come in rounds of kList; piece i of a round is at(i).  Loops are left rolled: this code stands between the launch
// and the first load, and a cold line of it costs more than its instructions.
template <int kDealers, int kList>
struct PagedDeal {
  static_assert((kList & (kList - 1)) == 0, "a power of two");
  int warp_sum[kDealers / 32][2];
  int first, last;         // ranks, among the units that have steps, of those in the share
  PagedRecord record;
  PagedPiece list[kList];

  struct Mine {            // of a thread: its units, and the width and the units with steps before them
    int u_begin, u_end, at, rank;
    int tail;              // rows of unit share * kDealers + thread, if there is one
  };
  // Rows of a unit: held (a word's distance every 32, as a thread's run of units lies together), or read again.
  __device__ __forceinline__ static int rows_of(const PagedArgs& a, const int* held, int u) {
    return held ? held[u + (u >> 5)] : paged_len(a, __ldcg(&a.state[u].x));
  }
  // Pieces of ranks [from, from + kList) go to the list; from < 0: all, and the ranks of the first and last and the record
  // are noted (if there are more than kList, round() fills the list again).
  __device__ __forceinline__ void fill(const PagedArgs& a, int window, int n_sink, const Mine& my, const PagedCut& cut, int share, int from,
                                       const int* held) {
    const int begin = cut.begin(share), end = cut.begin(share + 1);
    int r = my.rank, off = my.at;
#pragma unroll 1
    for (int u = my.u_begin; u < my.u_end; ++u) {
      const int len = rows_of(a, held, u), m = PagedSpan(len, window, n_sink).n;
      const int at = off + kPagedLead, lo = max(at, begin), hi = min(at + m, end);
      if (hi > lo) {
        // (divisions only for a unit that crosses the share's borders)
        const int f = at < begin ? cut.share_of(at) : share;
        const int l = at + m <= end ? share : cut.share_of(at + m - 1);
        const int parts = f == l ? 0 : l - f + 1, step = off - kPagedLead * r;
        if (from < 0) {
          if (off <= begin) first = r;         // a unit before it would reach past `begin`
          atomicMax(&last, r);
          if (parts > 0 && f == share) { record.u = u; record.slot = f + u; record.parts = parts; }
        }
        if (from < 0 || (r >= from && r < from + kList)) list[r & (kList - 1)] = PagedPiece{u, lo - at, hi - lo, len, step, f + u, parts};
      }
      off += m > 0 ? m + kPagedLead : 0;
      r += m > 0;
    }
  }
  __device__ __forceinline__ PagedCut start(const PagedArgs& a, int window, int n_sink, int share, Mine& my, int* held, bool copied_over) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid < kDealers && held)
#pragma unroll 4
      for (int u = tid; u < a.n_units; u += kDealers) held[u + (u >> 5)] = paged_len(a, __ldcg(&a.state[u].x));
    if (tid == 0) { first = 0; last = -1; record.parts = 0; }
    __syncthreads();
    my = Mine{};
    if (tid < kDealers) {
      const int chunk = (a.n_units + kDealers - 1) / kDealers;
      my.u_begin = min(a.n_units, tid * chunk);
      my.u_end = min(a.n_units, my.u_begin + chunk);
      int width = 0, units = 0;
#pragma unroll 1
      for (int u = my.u_begin; u < my.u_end; ++u) {
        const int m = PagedSpan(rows_of(a, held, u), window, n_sink).n;
        width += m > 0 ? m + kPagedLead : 0;
        units += m > 0;
      }
      my.at = width;
      my.rank = units;
#pragma unroll 1
      for (int off = 1; off < 32; off <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, my.at, off), tu = __shfl_up_sync(0xffffffffu, my.rank, off);
        if (lane >= off) { my.at += t; my.rank += tu; }
      }
      if (lane == 31) { warp_sum[warp][0] = my.at; warp_sum[warp][1] = my.rank; }
      my.at -= width;
      my.rank -= units;
    }
    __syncthreads();
    int total = 0, units = 0;
#pragma unroll
    for (int w = 0; w < kDealers / 32; ++w) {
      const int x = warp_sum[w][0], y = warp_sum[w][1];
      if (w < warp) { my.at += x; my.rank += y; }
      total += x;
      units += y;
    }
    const PagedCut cut(total, int(gridDim.x));
    if (tid == 0) record.steps = total - kPagedLead * units;
    if (tid < kDealers) fill(a, window, n_sink, my, cut, share, -1, held);
    const int u = share * kDealers + tid;
    if (tid < kDealers && u < a.n_units) my.tail = rows_of(a, held, u);
    if (copied_over) ptx::fence_proxy_async_smem();
    __syncthreads();
    return cut;
  }
  __device__ __forceinline__ int n_pieces() const { return last - first + 1; }
  // Before round rank0 / kList, by all threads.  The first is ready if all pieces fit.
  __device__ __forceinline__ void round(const PagedArgs& a, int window, int n_sink, const Mine& my, const PagedCut& cut, int share, int rank0) {
    if (n_pieces() <= kList) return;
    __syncthreads();
    if (threadIdx.x < kDealers) fill(a, window, n_sink, my, cut, share, first + rank0, nullptr);
    __syncthreads();
  }
  __device__ __forceinline__ const PagedPiece& at(int rank0, int i) const { return list[(first + rank0 + i) & (kList - 1)]; }
};
#endif

// Workspace: 256-byte header (word 0: sticky status); per share, how many partial results are there of the unit that
// runs from it into the next (zero between calls, and where they are whatever the cache, so that caches of any sizes can use
// one workspace in turn) and its record; row statistics (maximum in log2 units, sum) and unnormalised outputs of every
// (slot, head of the group); where weights are accumulated, the scores of every pool row in groups of 16 rows: [pool row / 16]
// [head of the group][16], in log2 units, and the records of the steps.
constexpr size_t kPagedHeaderBytes = 256;
struct PagedWs {
  int* status;
  int* tickets;
  PagedRecord* records;
  PagedStepRecord* steps;
  float2* ml;
  float* acc;
  float* score;
  size_t bytes;
};

}  // namespace tca
