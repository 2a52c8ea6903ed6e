// Attention of 32 query rows over a stream of 64-key tiles on the FP32 pipes, online softmax in one
// pass: the kernel for fp32 inputs (their tolerance rules out bf16 and tf32 products) and the slow
// cross-check of the tensor-core kernels.  Scores, statistics and accumulators are fp32.
//
// 256 threads in two groups of 128.  The groups take alternate key tiles, each with a softmax state of
// its own, and are merged at the end: a row's keys are then two chains half as long, which is what
// the longest row of a causal prompt, and a short cache, wait for.  Within a group thread (ty, tx) of the
// 8 x 16 grid holds scores of rows 4 ty .. 4 ty + 3 against keys tx, tx + 16, tx + 32, tx + 48 and output columns
// 4 tx + 64 c of the same rows, so both products run from shared memory with 16-byte loads (64 FMAs per 8
// loads; rows are padded by 16 bytes against bank conflicts).  K and V have one buffer each: the next
// K tile is fetched under this tile's softmax and second product, the next V tile under the next first
// product.  Bound by the FMA pipe and its operand loads.
#pragma once
#include <type_traits>

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "rowslice.cuh"

namespace tca {

constexpr int kSimtRows = 32, kSimtKeys = 64, kSimtThreads = 256, kSimtGroup = 128;

template <int D>
struct SimtSmem {
  static constexpr int kStride = D + 4;            // floats per row of Q, K, V
  static constexpr int kPStride = kSimtKeys + 4;
  static constexpr int kGroupFloats = 2 * kSimtKeys * kStride + kSimtRows * kPStride;   // K, V, P of a group
  static constexpr int kFloats = kSimtRows * kStride + 2 * kGroupFloats;
  static constexpr int kBytes = kFloats * 4;
  static constexpr int kCtasPerSm = D == 64 ? 2 : 1;
};

__device__ __forceinline__ void simt_group_sync(int group) {
  asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(kSimtGroup) : "memory");
}
// 16 bytes to shared memory, or zeros.
__device__ __forceinline__ void cp_async_16_or_zero(float* dst, const float* src, bool take) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
               ::"r"(ptx::smem_u32(dst)), "l"(src), "r"(take ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }

// kRows rows of D elements into shared memory by kThreads threads; rows >= n become zeros and are not read.
// fp32 rows go asynchronously (one commit group), bf16 rows are widened on the way.
template <typename T, int D, int kRows, int kThreads, typename RowPtr>
__device__ __forceinline__ void simt_load_rows(float* dst, int n, int tid, RowPtr row_ptr) {
  const T* any = row_ptr(0);
#pragma unroll 4
  for (int i = tid; i < kRows * (D / 4); i += kThreads) {
    const int r = i / (D / 4), c = (i % (D / 4)) * 4;
    float* to = dst + r * SimtSmem<D>::kStride + c;
    if constexpr (std::is_same<T, float>::value) {
      cp_async_16_or_zero(to, r < n ? row_ptr(r) + c : any, r < n);
    } else {
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < n) load4(row_ptr(r) + c, v);
      *reinterpret_cast<float4*>(to) = v;
    }
  }
  if constexpr (std::is_same<T, float>::value) cp_async_commit();
}

// Src: n_tiles(); n_rows(); q(r) -> const T*; keys(t) -> number of keys of tile t (1..64); k(t, r), v(t, r)
// -> const T*; last(t, r) -> index in tile t of the last key row r sees (< 0: none, never >= keys(t));
// masked(t): whether some row does not see all 64 keys of the tile.
// On return the threads of group 0 (threadIdx.x < 128; true is returned) hold the row maxima (in log2
// units), sums and unnormalised outputs of rows 4 ty .. 4 ty + 3, columns 4 tx + 64 c; m = -inf, l = 0,
// o = 0 for a row that saw nothing.
template <typename T, int D, typename Src>
__device__ __forceinline__ bool simt_flash(const Src& src, float scale_log2e, float* smem, float (&o)[4][D / 16],
                                           float (&m)[4], float (&l)[4]) {
  using S = SimtSmem<D>;
  constexpr int ST = S::kStride, PST = S::kPStride;
  const int group = threadIdx.x / kSimtGroup, tid = threadIdx.x % kSimtGroup;
  float* sQ = smem;
  float* sK = smem + kSimtRows * ST + group * S::kGroupFloats;
  float* sV = sK + kSimtKeys * ST;
  float* sP = sV + kSimtKeys * ST;
  const int tx = tid & 15, ty = tid >> 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o[i][c] = 0.f;
  }
  const int nt = src.n_tiles();
  auto load_k = [&](int t) {
    if (t < nt) simt_load_rows<T, D, kSimtKeys, kSimtGroup>(sK, src.keys(t), tid, [&](int r) { return src.k(t, r); });
    else cp_async_commit();                // keeps the count of pending groups
  };
  auto load_v = [&](int t) {
    if (t < nt) simt_load_rows<T, D, kSimtKeys, kSimtGroup>(sV, src.keys(t), tid, [&](int r) { return src.v(t, r); });
    else cp_async_commit();
  };
  __syncthreads();                         // the buffers may still be read by the item before
  simt_load_rows<T, D, kSimtRows, kSimtThreads>(sQ, src.n_rows(), threadIdx.x, [&](int r) { return src.q(r); });
  load_k(group);
  load_v(group);
  cp_async_wait<2>();
  __syncthreads();                         // Q is shared by the groups
  for (int t = group; t < nt; t += 2) {
    cp_async_wait<1>();                    // K of this tile; V may still be on its way
    simt_group_sync(group);
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
    simt_group_sync(group);                // K has been read
    load_k(t + 2);
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
    cp_async_wait<1>();                    // V of this tile; the next K may still be on its way
    simt_group_sync(group);                // (P needs no more than a warp: a row's 16 threads are half of one)
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
    simt_group_sync(group);                // V has been read
    load_v(t + 2);
  }
  cp_async_wait<0>();
  // group 1 hands its state over through group 1's own buffers
  float* sO = smem + kSimtRows * ST + S::kGroupFloats;
  float* sM = sO + kSimtRows * ST;
  if (group == 1) {
    simt_group_sync(group);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        *reinterpret_cast<float4*>(sO + (ty * 4 + i) * ST + tx * 4 + 64 * c) =
            make_float4(o[i][c * 4], o[i][c * 4 + 1], o[i][c * 4 + 2], o[i][c * 4 + 3]);
      if (tx == 0) {
        sM[2 * (ty * 4 + i)] = m[i];
        sM[2 * (ty * 4 + i) + 1] = l[i];
      }
    }
  }
  __syncthreads();
  if (group == 1) return false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float m1 = sM[2 * (ty * 4 + i)], l1 = sM[2 * (ty * 4 + i) + 1];
    const float mn = fmaxf(m[i], m1), base = (mn == -INFINITY) ? 0.f : mn;
    const float w0 = exp2f(m[i] - base), w1 = exp2f(m1 - base);
    l[i] = l[i] * w0 + l1 * w1;
    m[i] = mn;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      const float4 v = *reinterpret_cast<const float4*>(sO + (ty * 4 + i) * ST + tx * 4 + 64 * c);
      o[i][c * 4 + 0] = o[i][c * 4 + 0] * w0 + v.x * w1;
      o[i][c * 4 + 1] = o[i][c * 4 + 1] * w0 + v.y * w1;
      o[i][c * 4 + 2] = o[i][c * 4 + 2] * w0 + v.z * w1;
      o[i][c * 4 + 3] = o[i][c * 4 + 3] * w0 + v.w * w1;
    }
  }
  return true;
}

}  // namespace tca
