// Compression of the block that leaves the window while tokens are appended (Section 4.2, "Online
// Token Selection in Decoding Stage"), shared by the calls that append: score the b oldest keys of
// a unit's ring with the current query group (Eq. 5 restricted to the block, fp64), keep the top
// t_keep by the order the prefill uses, and move those rows to the end of the global
// region in ascending position.
#pragma once
#include <type_traits>

#include "common.cuh"
#include "rowslice.cuh"

namespace tca {

constexpr int kCompressThreads = 256;   // CTA size of every kernel that calls this
static_assert(kCompressThreads == 2 * kMaxBlock, "two threads per key of a block");

// Scores of the b oldest ring rows against the G queries, fp64, into xs; D = 16 EPL.  16 lanes per row, EPL adjacent
// elements each, added in the order of the elements and then across the lanes.  What bounds it is latency (an
// fp64 multiply-add takes 28 clocks, its unit starts a warp's every other clock), so kRows rows times kHeads
// heads run side by side and go through the reduction across the lanes together (a transposing butterfly:
// the same pairs in the same order as one by one), and the next keys are on their way meanwhile.  A key is
// converted once for kHeads heads.  The queries lie in shared memory as fp64, element e of lane l at e * 16 + l:
// without bank conflicts.  A block of 128 keys and 4 heads: 7.4 thousand clocks (with conflicts, 4 rows
// x 1 head and no keys ahead 22.8).
// G is a multiple of kHeads.
template <typename T, int EPL, int kRows, int kHeads>
__device__ __forceinline__ void block_logits(const T* __restrict__ q_unit, int64_t q_stride, const T* __restrict__ Kc, int64_t ring,
                                             int64_t tail_head, int64_t tail_cap, int G, int b, double sm_scale,
                                             double* qs, double (*xs)[kMaxBlock]) {
  constexpr int D = 16 * EPL, kGroups = kCompressThreads / 16, N = kRows * kHeads;
  static_assert(N == 4 || N == 8, "values of a butterfly over 16 lanes");
  const int tid = threadIdx.x, lane16 = tid & 15, grp = tid >> 4;
  RowF<T, EPL> next[kRows];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int s = 0; s < kRows; ++s) {
      int64_t slot = tail_head + min(i0 + s * kGroups + grp, b - 1);
      if (slot >= tail_cap) slot -= tail_cap;
      next[s].load_cached(Kc + (ring + slot) * D + lane16 * EPL);
    }
  };
  fetch(0);
  for (int i = tid; i < G * D; i += kCompressThreads) {
    const int g = i / D, c = i % D;
    qs[g * D + (c % EPL) * 16 + c / EPL] = double(elt_to_float(q_unit[g * q_stride + c]));
  }
  __syncthreads();
#pragma unroll 1
  for (int i0 = 0; i0 < b; i0 += kGroups * kRows) {
    double kd[kRows][EPL];
#pragma unroll
    for (int s = 0; s < kRows; ++s)
#pragma unroll
      for (int e = 0; e < EPL; ++e) kd[s][e] = next[s].get(e);
    if (i0 + kGroups * kRows < b) fetch(i0 + kGroups * kRows);
#pragma unroll 1
    for (int g0 = 0; g0 < G; g0 += kHeads) {
      double acc[N];                       // value s * kHeads + h: row s, head g0 + h
#pragma unroll
      for (int n = 0; n < N; ++n) acc[n] = 0.0;
#pragma unroll
      for (int e = 0; e < EPL; ++e)
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
          const double qe = qs[(g0 + h) * D + e * 16 + lane16];
#pragma unroll
          for (int s = 0; s < kRows; ++s) acc[s * kHeads + h] = fma(qe, kd[s][e], acc[s * kHeads + h]);
        }
      // each exchange halves the values a lane holds and doubles the lanes in them; then plain sums
      int n = 0;                           // the value that ends up in this lane
#pragma unroll
      for (int off = 8, half = N / 2; off > 0; off >>= 1, half >>= 1) {
        const bool up = lane16 & off;
        if (half >= 1) {
#pragma unroll
          for (int j = 0; j < half; ++j) acc[j] = (up ? acc[j + half] : acc[j]) + shfl_xor_double(up ? acc[j] : acc[j + half], off);
          n += up ? half : 0;
        } else {
          acc[0] += shfl_xor_double(acc[0], off);
        }
      }
      const int i = i0 + n / kHeads * kGroups + grp, g = g0 + n % kHeads;
      if ((lane16 & (16 / N - 1)) == 0 && i < b) xs[g][i] = acc[0] * sm_scale;
    }
  }
}

// Called by the whole CTA.  q_unit: query of the unit's first head, q_stride elements to the next
// head's.  The rows must be visible to the CTA (a barrier after they were written); on return the
// moved rows have been written but not yet synchronised.
template <typename T>
__device__ __forceinline__ void compress_oldest_block(const T* __restrict__ q_unit, int64_t q_stride, T* __restrict__ Kc,
                                                      T* __restrict__ Vc, int32_t* __restrict__ pos, int64_t seg,
                                                      int64_t ring, int64_t n_global, int64_t tail_head,
                                                      int64_t tail_cap, int t_keep, int D, int G, int b,
                                                      double sm_scale) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // ---- logits of the b oldest tail tokens against the G current queries, fp64
  __shared__ double xs[kMaxGroup][kMaxBlock];
  __shared__ double lse[kMaxGroup];
  __shared__ double qs[kMaxGroup * 128];           // head_dim is 64 or 128
  __shared__ int kept_slot[kMaxBlock];
  __shared__ unsigned long long keys[kMaxBlock];
  __shared__ int ranks[kMaxBlock], rank_sum[kCompressThreads / 32];
  __shared__ unsigned kept_mask[kMaxBlock / 32];
  // Four heads at once if they come in fours (128 units that compress 128 keys each, 4 heads: 10.2 us against 10.6
  // with one at a time, 8 heads: 12.7 against 12.9; 3 heads: 10.3 against 10.1, 5 heads: 12.8 against 11.3).
  auto logits = [&](auto epl) {
    constexpr int EPL = decltype(epl)::value;
    if (G % 4 == 0) block_logits<T, EPL, 2, 4>(q_unit, q_stride, Kc, ring, tail_head, tail_cap, G, b, sm_scale, qs, xs);
    else block_logits<T, EPL, 4, 1>(q_unit, q_stride, Kc, ring, tail_head, tail_cap, G, b, sm_scale, qs, xs);
  };
  if (D == 128) logits(std::integral_constant<int, 8>{});
  else logits(std::integral_constant<int, 4>{});
  __syncthreads();
  if (warp < G) {  // log-sum-exp of head `warp` over the block
    double mx = -1.0e308;
#pragma unroll 4
    for (int i = lane; i < b; i += 32) mx = fmax(mx, xs[warp][i]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) mx = fmax(mx, shfl_xor_double(mx, off));
    double sum = 0.0;
#pragma unroll 4
    for (int i = lane; i < b; i += 32) sum += exp(xs[warp][i] - mx);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += shfl_xor_double(sum, off);
    if (lane == 0) lse[warp] = mx + log(sum);
  }
  __syncthreads();
  if (tid < b) {   // score of key `tid`: the mean over the group, in logs (the 1/G is common to all)
    double score;
    if (G == 1) {
      score = xs[0][tid] - lse[0];
    } else {
      double top = -1.0e308;
      for (int g = 0; g < G; ++g) top = fmax(top, xs[g][tid] - lse[g]);
      double sum = 0.0;
#pragma unroll 4
      for (int g = 0; g < G; ++g) sum += exp(xs[g][tid] - lse[g] - top);
      score = top + log(sum);
    }
    keys[tid] = ordered_key(score);
  }
  __syncthreads();
  // Top t_keep by rank: a key's rank is the number of larger keys and of equal ones at lower indices, the
  // set the radix select of the prefill keeps.  With one block per CTA the b^2 comparisons (two threads per
  // key, half of them each) take less than its 50 or so dependent rounds.  The larger ones are counted first:
  // if that adds up to b (b - 1) / 2 no two keys are equal, and it is done.
  {
    const int i = tid & (kMaxBlock - 1), half = tid / kMaxBlock;
    const int j0 = half * (b / 2), j1 = half == 0 ? b / 2 : b;
    const unsigned long long mine = i < b ? keys[i] : ~0ull;
    int rank = 0;
#pragma unroll 8
    for (int j = j0; j < j1; ++j) rank += keys[j] > mine ? 1 : 0;
    const int sum = __reduce_add_sync(0xffffffffu, rank);
    if (lane == 0) rank_sum[warp] = sum;
    if (half == 1) ranks[i] = rank;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kCompressThreads / 32; ++w) all += rank_sum[w];
    if (all != b * (b - 1) / 2) {          // the same for all threads
#pragma unroll 1
      for (int j = j0; j < min(i, j1); ++j) rank += keys[j] == mine ? 1 : 0;
      __syncthreads();
      if (half == 1) ranks[i] = rank;
      __syncthreads();
    }
    if (half == 0) {
      const bool keep = i < b && rank + ranks[i] < t_keep;
      const unsigned bal = __ballot_sync(0xffffffffu, keep);
      if (lane == 0) kept_mask[warp] = bal;
      __syncwarp();
    }
    __syncthreads();
    if (half == 0 && ((kept_mask[warp] >> lane) & 1u)) {
      int before = __popc(kept_mask[warp] & ((1u << lane) - 1u));
      for (int w = 0; w < warp; ++w) before += __popc(kept_mask[w]);
      kept_slot[before] = i;
    }
  }
  __syncthreads();
  // ---- move the kept rows to the end of the global region (ring and region are disjoint)
  int kept_pos = 0;
  if (tid < t_keep) {
    int64_t slot = tail_head + kept_slot[tid];
    if (slot >= tail_cap) slot -= tail_cap;
    kept_pos = pos[ring + slot];
  }
  // 16-byte pieces, four rows' worth in flight per thread
  const int shift = 31 - __clz(D * int(sizeof(T)) / 16);
  const int n_pieces = t_keep << shift;
  uint4* K4 = reinterpret_cast<uint4*>(Kc);
  uint4* V4 = reinterpret_cast<uint4*>(Vc);
  for (int i0 = tid; i0 < n_pieces; i0 += 4 * kCompressThreads) {
    uint4 kv[4], vv[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + j * kCompressThreads;
      if (i >= n_pieces) continue;
      int64_t slot = tail_head + kept_slot[i >> shift];
      if (slot >= tail_cap) slot -= tail_cap;
      const int64_t src = ((ring + slot) << shift) + (i & ((1 << shift) - 1));
      kv[j] = K4[src];
      vv[j] = V4[src];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + j * kCompressThreads;
      if (i >= n_pieces) continue;
      const int64_t dst = ((seg + n_global) << shift) + i;
      K4[dst] = kv[j];
      V4[dst] = vv[j];
    }
  }
  if (tid < t_keep) pos[seg + n_global + tid] = kept_pos;
}

}  // namespace tca
