// Attention of 64 query rows over a stream of 64-key tiles on the FP32 pipes, online softmax in one
// pass: the kernel for fp32 inputs (their tolerance rules out bf16 and tf32 products) and the slow
// cross-check of the tensor-core kernels.  Scores, statistics and accumulators are fp32.
//
// 256 threads; thread (ty, tx) of the 16 x 16 grid holds scores of rows 4 ty .. 4 ty + 3 against keys
// tx, tx + 16, tx + 32, tx + 48 and output columns 4 tx + 64 c of the same rows, so both products run
// from shared memory with 16-byte loads: 64 FMAs per 8 loads for the scores, 32 D/16 per 4 + 4 D/64
// for the output.  Rows are padded by 16 bytes against bank conflicts.
#pragma once
#include "common.cuh"
#include "rowslice.cuh"

#include <type_traits>

namespace tca {

constexpr int kSimtRows = 64, kSimtKeys = 64, kSimtThreads = 256;

template <int D>
struct SimtSmem {
  static constexpr int kStride = D + 4;            // floats per row of Q, K, V
  static constexpr int kPStride = kSimtKeys + 4;
  static constexpr int kFloats = 3 * 64 * kStride + kSimtRows * kPStride;
  static constexpr int kBytes = kFloats * 4;
};

// 64 rows of D elements into shared memory; rows >= n become zeros and are not read.
template <typename T, int D, typename RowPtr>
__device__ __forceinline__ void simt_load_rows(float* dst, int n, RowPtr row_ptr) {
#pragma unroll 4
  for (int i = threadIdx.x; i < 64 * (D / 4); i += kSimtThreads) {
    const int r = i / (D / 4), c = (i % (D / 4)) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < n) load4(row_ptr(r) + c, v);
    *reinterpret_cast<float4*>(dst + r * SimtSmem<D>::kStride + c) = v;
  }
}

// Src: n_tiles(); n_rows(); q(r) -> const T*; keys(t) -> number of keys of tile t (1..64); k(t, r), v(t, r)
// -> const T*; last(t, r) -> index in tile t of the last key row r sees (< 0: none, never >= keys(t));
// masked(t): whether some row does not see all 64 keys of the tile.
// On return m, l and o hold the row maxima (in log2 units), sums and unnormalised outputs of this
// thread's rows; m = -inf, l = 0, o = 0 for a row that saw nothing.
template <typename T, int D, typename Src>
__device__ __forceinline__ void simt_flash(const Src& src, float scale_log2e, float* smem, float (&o)[4][D / 16],
                                           float (&m)[4], float (&l)[4]) {
  constexpr int ST = SimtSmem<D>::kStride, PST = SimtSmem<D>::kPStride;
  float* sQ = smem;
  float* sK = sQ + 64 * ST;
  float* sV = sK + 64 * ST;
  float* sP = sV + 64 * ST;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o[i][c] = 0.f;
  }
  simt_load_rows<T, D>(sQ, src.n_rows(), [&](int r) { return src.q(r); });
  const int nt = src.n_tiles();
  for (int t = 0; t < nt; ++t) {
    __syncthreads();                       // the previous tile has been consumed
    const int n = src.keys(t);
    simt_load_rows<T, D>(sK, n, [&](int r) { return src.k(t, r); });
    simt_load_rows<T, D>(sV, n, [&](int r) { return src.v(t, r); });
    __syncthreads();
    float s[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
    for (int d = 0; d < D; d += 4) {
      float4 q[4], k[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const float4*>(sQ + (ty * 4 + i) * ST + d);
#pragma unroll
      for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const float4*>(sK + (tx + 16 * j) * ST + d);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          s[i][j] = fmaf(q[i].w, k[j].w, fmaf(q[i].z, k[j].z, fmaf(q[i].y, k[j].y, fmaf(q[i].x, k[j].x, s[i][j]))));
    }
    const bool masked = src.masked(t);
    int last[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      last[i] = masked ? src.last(t, ty * 4 + i) : kSimtKeys - 1;
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = (tx + 16 * j <= last[i]) ? s[i][j] * scale_log2e : -INFINITY;   // a masked score counts for nothing
        mx = fmaxf(mx, s[i][j]);
      }
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
      const float m_new = fmaxf(m[i], mx);
      const float base = (m_new == -INFINITY) ? 0.f : m_new;    // nothing seen yet: every weight is exp2(-inf) = 0
      const float corr = exp2f(m[i] - base);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = exp2f(s[i][j] - base);
        sum += s[i][j];
        sP[(ty * 4 + i) * PST + tx + 16 * j] = s[i][j];
      }
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      l[i] = l[i] * corr + sum;
      m[i] = m_new;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[i][c] *= corr;
    }
    __syncwarp();                          // a row's 16 threads are half a warp: P needs no wider barrier
    auto accumulate = [&](auto guarded) {
#pragma unroll 2
      for (int kk = 0; kk < kSimtKeys; kk += 4) {
        float4 p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = *reinterpret_cast<const float4*>(sP + (ty * 4 + i) * PST + kk);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            const float4 v = *reinterpret_cast<const float4*>(sV + (kk + e) * ST + tx * 4 + 64 * c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float pe = e == 0 ? p[i].x : e == 1 ? p[i].y : e == 2 ? p[i].z : p[i].w;
              // a key the row does not see must not reach it even if its value is an infinity or a NaN
              if (!decltype(guarded)::value || kk + e <= last[i]) {
                o[i][c * 4 + 0] = fmaf(pe, v.x, o[i][c * 4 + 0]);
                o[i][c * 4 + 1] = fmaf(pe, v.y, o[i][c * 4 + 1]);
                o[i][c * 4 + 2] = fmaf(pe, v.z, o[i][c * 4 + 2]);
                o[i][c * 4 + 3] = fmaf(pe, v.w, o[i][c * 4 + 3]);
              }
            }
          }
        }
      }
    };
    if (masked) accumulate(std::true_type{}); else accumulate(std::false_type{});
  }
}

}  // namespace tca
