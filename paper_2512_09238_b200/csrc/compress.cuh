// Compression of the block that leaves the window while tokens are appended (Section 4.2, "Online
// Token Selection in Decoding Stage"), shared by the calls that append: score the b oldest keys of
// a unit's ring with the current query group (Eq. 5 restricted to the block, fp64), keep the top
// t_keep by the order the prefill uses, and move those rows to the end of the global
// region in ascending position.
#pragma once
#include "common.cuh"
#include "rowslice.cuh"

namespace tca {

constexpr int kCompressThreads = 256;   // CTA size of every kernel that calls this
static_assert(kCompressThreads == 2 * kMaxBlock, "two threads per key of a block");

// Called by the whole CTA.  q_unit: query of the unit's first head, q_stride elements to the next
// head's.  The rows must be visible to the CTA (a barrier after they were written); on return the
// moved rows have been written but not yet synchronised.
template <typename T>
__device__ __forceinline__ void compress_oldest_block(const T* __restrict__ q_unit, int64_t q_stride, T* __restrict__ Kc,
                                                      T* __restrict__ Vc, int32_t* __restrict__ pos, int64_t seg,
                                                      int64_t ring, int64_t n_global, int64_t tail_head,
                                                      int64_t tail_cap, int t_keep, int D, int G, int b,
                                                      double sm_scale) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lane16 = tid & 15, grp = tid >> 4;
  // ---- logits of the b oldest tail tokens against the G current queries, fp64
  __shared__ double xs[kMaxGroup][kMaxBlock];
  __shared__ double lse[kMaxGroup];
  __shared__ int kept_slot[kMaxBlock];
  __shared__ unsigned long long keys[kMaxBlock];
  __shared__ int ranks[kMaxBlock];
  __shared__ unsigned kept_mask[kMaxBlock / 32];
  // 16 lanes per row, D/16 adjacent elements each, added in the order of the elements and then across the
  // lanes.  What bounds this is the conversion to fp64 (a quarter of the FMA rate), so the queries are
  // converted once, into shared memory, and a key once for all heads; four rows go through the reduction
  // across the lanes together (a transposing butterfly, the same pairs in the same order as row by row).
  // One block of 128 keys, 4 heads: 22.5 thousand clocks with a conversion per factor and a reduction per row.
  __shared__ double qs[kMaxGroup * kMaxBlock];     // head_dim <= 128
  static_assert(kMaxBlock >= 128, "a query per row of qs");
  for (int i = tid; i < G * D; i += kCompressThreads) qs[i] = double(elt_to_float(q_unit[(i / D) * q_stride + i % D]));
  __syncthreads();
  const int EPL = D / 16;
  constexpr int kGroups = kCompressThreads / 16, kBatch = 4;
  for (int i0 = 0; i0 < b; i0 += kGroups * kBatch) {
    double kd[kBatch][8];
#pragma unroll
    for (int s = 0; s < kBatch; ++s) {
      int64_t slot = tail_head + min(i0 + s * kGroups + grp, b - 1);
      if (slot >= tail_cap) slot -= tail_cap;
      const T* krow = Kc + (ring + slot) * D + lane16 * EPL;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
        if (h * 4 < EPL) load4(krow + h * 4, f);
        kd[s][h * 4] = f.x; kd[s][h * 4 + 1] = f.y; kd[s][h * 4 + 2] = f.z; kd[s][h * 4 + 3] = f.w;
      }
    }
#pragma unroll 1
    for (int g = 0; g < G; ++g) {
      const double* qrow = qs + g * D + lane16 * EPL;
      double acc[kBatch] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e >= EPL) continue;
        const double qe = qrow[e];
#pragma unroll
        for (int s = 0; s < kBatch; ++s) acc[s] = fma(qe, kd[s][e], acc[s]);
      }
      const bool up8 = lane16 & 8, up4 = lane16 & 4;
      const double r0 = (up8 ? acc[2] : acc[0]) + shfl_xor_double(up8 ? acc[0] : acc[2], 8);
      const double r1 = (up8 ? acc[3] : acc[1]) + shfl_xor_double(up8 ? acc[1] : acc[3], 8);
      double r = (up4 ? r1 : r0) + shfl_xor_double(up4 ? r0 : r1, 4);
      r += shfl_xor_double(r, 2);
      r += shfl_xor_double(r, 1);
      const int i = i0 + ((up8 ? 2 : 0) + (up4 ? 1 : 0)) * kGroups + grp;   // the row whose total ends up here
      if ((lane16 & 3) == 0 && i < b) xs[g][i] = r * sm_scale;
    }
  }
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
  // key, half of them each) take a quarter of the time of its 50 or so dependent rounds.
  {
    const int i = tid & (kMaxBlock - 1), half = tid / kMaxBlock;
    int rank = 0;
    if (i < b) {
      const unsigned long long mine = keys[i];
      const int j0 = half * (b / 2), j1 = half == 0 ? b / 2 : b;
#pragma unroll 8
      for (int j = j0; j < j1; ++j) rank += (keys[j] > mine || (keys[j] == mine && j < i)) ? 1 : 0;
    }
    if (half == 1) ranks[i] = rank;
    __syncthreads();
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
  if (tid < t_keep) {
    int64_t slot = tail_head + kept_slot[tid];
    if (slot >= tail_cap) slot -= tail_cap;
    pos[seg + n_global + tid] = pos[ring + slot];
  }
}

}  // namespace tca
