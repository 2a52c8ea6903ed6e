// The paged cache: which slots a new token sees, how the visible rows of all units are dealt to CTAs, and the layout of
// the partial results of tca_attn_paged.
#pragma once
#include "common.cuh"

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

// How the steps of all units are dealt: laid end to end they are cut into equal shares, one per CTA, wherever the
// cuts fall; a share that runs into the next unit works on both.  A unit counts `lead` steps more than it has, which
// is what starting on one costs.  The cuts follow from the device's state, so a captured launch stays right when the
// cache has changed since.  Pair (share i, unit u) has partial slot i + u: pairs advance in one of the two at a time.
struct PagedPlan {
  int n_shares, min_share, lead;
};
struct PagedPiece {
  int u, s0, n, whole;     // steps [s0, s0 + n) of unit u; whole: all it has
  int len;                 // rows of the unit
};

#ifdef __CUDACC__
// All threads of the CTA deal together (a thread takes a run of units, the CTA scans their sums): one trip to memory
// for up to kThreads units.  Pieces come in rounds of kList.
template <int kThreads, int kList>
struct PagedDeal {
  int warp_sum[kThreads / 32][2];
  int first_rank, n_pieces;
  PagedPiece list[kList];

  __device__ __forceinline__ static int share_of(int x, int q, int longer) {   // the share that holds step x
    const int head = longer * (q + 1);
    return x < head ? x / (q + 1) : longer + (x - head) / q;
  }
  // Fills the list with the share's pieces of ranks [rank0, rank0 + kList) and returns how many pieces it has in
  // all.  table: where each unit's partial results lie (written by the share that holds its first step); null: not.
  __device__ int deal(const PagedArgs& a, const PagedPlan& plan, int window, int n_sink, int share, int rank0, int2* table) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int chunk = (a.n_units + kThreads - 1) / kThreads;
    const int u_begin = tid * chunk, u_end = min(a.n_units, u_begin + chunk);
    int steps = 0, units = 0;
    int len = 0, one = 0;              // rows and steps of the only unit, if there is one
    for (int u = u_begin; u < u_end; ++u) {
      len = paged_len(a, a.state[u].x);
      one = PagedSpan(len, window, n_sink).n;
      steps += one > 0 ? one + plan.lead : 0;
      units += one > 0;
    }
    int incl = steps, incl_u = units;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, incl, off), tu = __shfl_up_sync(0xffffffffu, incl_u, off);
      if (lane >= off) { incl += t; incl_u += tu; }
    }
    __syncthreads();                   // the list and the sums may still be read from the round before
    if (lane == 31) { warp_sum[warp][0] = incl; warp_sum[warp][1] = incl_u; }
    if (tid == 0) { n_pieces = 0; first_rank = 0; }
    __syncthreads();
    int at = incl - steps, rank = incl_u - units, total = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) { at += warp_sum[w][0]; rank += warp_sum[w][1]; }
      total += warp_sum[w][0];
    }
    const int n = max(1, min(plan.n_shares, total / plan.min_share));
    const int q = total / n, longer = total - q * n;
    const int begin = share < n ? share * q + min(share, longer) : total;
    const int end = share < n ? begin + q + (share < longer ? 1 : 0) : total;
    for (int pass = 0; pass < 2; ++pass) {
      // first which of the units comes first in the share, then the list
      int off = at, r = rank;
      for (int u = u_begin; u < u_end; ++u) {
        if (off >= end) break;
        int m = one;
        if (chunk > 1) {
          len = paged_len(a, a.state[u].x);
          m = PagedSpan(len, window, n_sink).n;
        }
        if (m == 0) continue;
        const int rows = off + plan.lead;                  // where the unit's own steps begin
        const int lo = max(rows, begin), hi = min(rows + m, end);
        if (hi > lo) {
          if (pass == 0) {
            if (off <= begin) first_rank = r;
            atomicAdd(&n_pieces, 1);
          } else {
            const int i = r - first_rank - rank0;
            if (i >= 0 && i < kList) list[i] = PagedPiece{u, lo - rows, hi - lo, hi - lo == m, len};
            if (table && lo == rows)
              table[u] = make_int2(share + u, hi - lo == m ? 0 : share_of(rows + m - 1, q, longer) - share + 1);
          }
        }
        off += m + plan.lead;
        ++r;
      }
      __syncthreads();
    }
    return n_pieces;
  }
};
#endif

// Workspace: 256-byte header (word 0: sticky status), where each unit's partial results lie (first slot, number; 0: its
// only share wrote the result itself), row statistics (maximum in log2 units, sum) and unnormalised outputs of every
// (slot, head of the group); where weights are accumulated, the scores of every pool row in groups of 16 rows:
// [pool row / 16][head of the group][16], in log2 units.
constexpr size_t kPagedHeaderBytes = 256;
struct PagedWs {
  int* status;
  int2* table;
  float2* ml;
  float* acc;
  float* score;
  size_t bytes;
};

}  // namespace tca
