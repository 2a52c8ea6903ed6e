// Compression of the block that leaves the window while tokens are appended (Section 4.2, "Online
// Token Selection in Decoding Stage"), shared by the calls that append: score the b oldest keys of
// a unit's ring with the current query group (Eq. 5 restricted to the block, fp64), keep the top
// t_keep by the same radix select the prefill uses, and move those rows to the end of the global
// region in ascending position.
#pragma once
#include "common.cuh"
#include "rowslice.cuh"

namespace tca {

constexpr int kCompressThreads = 256;   // CTA size of every kernel that calls this

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
  const int EPL = D / 16;
  for (int i0 = 0; i0 < b; i0 += kCompressThreads / 16) {  // uniform trip count: shuffles below need whole warps
    const int i = min(i0 + grp, b - 1);
    int64_t slot = tail_head + i;
    if (slot >= tail_cap) slot -= tail_cap;
    const T* krow = Kc + (ring + slot) * D + lane16 * EPL;
    for (int g = 0; g < G; ++g) {
      const T* qrow = q_unit + g * q_stride + lane16 * EPL;
      double acc = 0.0;
      for (int e = 0; e < EPL; ++e) acc = fma(double(elt_to_float(qrow[e])), double(elt_to_float(krow[e])), acc);
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) acc += shfl_xor_double(acc, off);
      if (lane16 == 0 && i0 + grp < b) xs[g][i] = acc * sm_scale;
    }
  }
  __syncthreads();
  if (warp < G) {  // log-sum-exp of head `warp` over the block
    double mx = -1.0e308;
    for (int i = lane; i < b; i += 32) mx = fmax(mx, xs[warp][i]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) mx = fmax(mx, shfl_xor_double(mx, off));
    double sum = 0.0;
    for (int i = lane; i < b; i += 32) sum += exp(xs[warp][i] - mx);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += shfl_xor_double(sum, off);
    if (lane == 0) lse[warp] = mx + log(sum);
  }
  __syncthreads();
  if (warp == 0) {
    unsigned long long key[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int i = s * 32 + lane;
      double score = -1.0e308;
      if (i < b) {
        if (G == 1) {
          score = xs[0][i] - lse[0];
        } else {
          double top = -1.0e308;
          for (int g = 0; g < G; ++g) top = fmax(top, xs[g][i] - lse[g]);
          double sum = 0.0;
          for (int g = 0; g < G; ++g) sum += exp(xs[g][i] - lse[g] - top);
          score = top + log(sum);
        }
      }
      key[s] = ordered_key(score);
    }
    const unsigned keep = radix_select_top_t(key, b, t_keep, lane);
    int before = 0;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const bool k = (keep >> s) & 1u;
      const unsigned bal = __ballot_sync(0xffffffffu, k);
      if (k) kept_slot[before + __popc(bal & ((1u << lane) - 1u))] = s * 32 + lane;
      before += __popc(bal);
    }
  }
  __syncthreads();
  // ---- move the kept rows to the end of the global region (ring and region are disjoint)
  for (int i = tid; i < t_keep * D; i += kCompressThreads) {
    const int r = i / D, e = i - r * D;
    int64_t slot = tail_head + kept_slot[r];
    if (slot >= tail_cap) slot -= tail_cap;
    Kc[(seg + n_global + r) * D + e] = Kc[(ring + slot) * D + e];
    Vc[(seg + n_global + r) * D + e] = Vc[(ring + slot) * D + e];
    if (e == 0) pos[seg + n_global + r] = pos[ring + slot];
  }
}

}  // namespace tca
