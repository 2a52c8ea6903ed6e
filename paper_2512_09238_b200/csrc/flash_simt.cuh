// Attention of a block of query rows over a stream of key tiles on the FP32 pipes, online softmax in one
// pass: the kernel for fp32 inputs (their tolerance rules out a single bf16 or tf32 product) and the slow
// cross-check of the tensor-core kernels.  Scores, statistics and accumulators are fp32.
//
// 256 threads in two groups of 128.  The groups take alternate key tiles, each with a softmax state of
// its own, and are merged at the end: a row's keys are then two chains half as long, which is what
// the longest row of a causal prompt, and a short cache, wait for.  Within a group thread (ty, tx) of the
// 8 x 16 grid holds scores of rows RT ty .. against keys tx, tx + 16, ... (KT of them) and output columns
// 4 tx + 64 c of the same rows; both products run from shared memory with 16-byte loads (rows are padded by
// 16 bytes against bank conflicts).  K and V have one buffer each: the next K tile is fetched under this
// tile's softmax and second product, the next V tile under the next first product.
//
// What bounds it is the shared-memory pipe, four clocks per warp for a 16-byte load against one clock of a
// scheduler for an FMA: 4 x 4 scores per thread take 8 loads (32 clocks of the SM) per 64 FMAs (16), 8 x 4 take 12
// (48) per 128 (32).  So there are two shapes: SimtSmall for few rows and short prompts, SimtLarge where there is
// work for all SMs in tiles of 64 rows (fp32 prompt of 2K, 8 heads of 64: 149 -> 139 us, 31 TFLOP/s).
//
// A row's result must not depend on which shape the batch around it led to.  So both take 64 keys at a time and
// deal them to the groups in the same way (8 x 8 scores and 128 keys for head_dim 64 took 138 us, and 142 with
// its keys in the order of the others), and what the compiler could contract into a multiply-add in one shape and
// not in the other is written out.
#pragma once
#include <type_traits>

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "rowslice.cuh"

namespace tca {

constexpr int kSimtThreads = 256, kSimtGroup = 128;

// RT rows and KT keys per thread.
template <int RT_, int KT_>
struct SimtShape {
  static constexpr int RT = RT_, KT = KT_;
  static constexpr int kRows = 8 * RT, kKeys = 16 * KT;
};
using SimtSmall = SimtShape<4, 4>;
using SimtLarge = SimtShape<8, 4>;
static_assert(SimtSmall::kKeys == SimtLarge::kKeys, "a row's keys are taken in the same order whatever the shape");

template <int D, typename Shape>
struct SimtSmem {
  static constexpr int kStride = D + 4;            // floats per row of Q, K, V
  static constexpr int kPStride = Shape::kKeys + 4;
  static constexpr int kGroupFloats = 2 * Shape::kKeys * kStride + Shape::kRows * kPStride;   // K, V, P of a group
  static constexpr int kFloats = Shape::kRows * kStride + 2 * kGroupFloats;
  static constexpr int kBytes = kFloats * 4;
  static constexpr int kCtasPerSm = kBytes <= 113 * 1024 ? 2 : 1;
  static_assert(kBytes <= 227 * 1024, "shared memory");
};

__device__ __forceinline__ void simt_group_sync(int group) {
  asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(kSimtGroup) : "memory");
}
__device__ __forceinline__ bool simt_group_any(int group, bool p) {
  int any;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.or.pred q, %2, %3, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
               : "=r"(any) : "r"(int(p)), "r"(group + 1), "n"(kSimtGroup) : "memory");
  return any != 0;
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
  constexpr int kPieces = D / 4, kStep = kThreads / kPieces;    // a thread keeps its column and walks down the rows
  const int c = (tid % kPieces) * 4, r0 = tid / kPieces;
  const T* any = row_ptr(0);
#pragma unroll 8
  for (int r = r0; r < kRows; r += kStep) {
    float* to = dst + r * (D + 4) + c;
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

// Src: n_tiles(); n_rows(); q(r) -> const T*; keys(t) -> number of keys of tile t (1..kKeys); k(t), v(t)
// -> const T*, its first row, k_stride(), v_stride() elements to the next; last(t, r) -> index in tile t of the last key row r sees (< 0: none, never >= keys(t));
// masked(t): whether some row does not see all kKeys keys of the tile.  kGap: a tile's keys need not lie together (k(t, r), v(t, r)
// -> its row r); rows also do not see keys [gap_begin(t), gap_end(t, r)) of it, and all see those from sink_begin(t) on; a
// masked tile whose values are all finite is accumulated without looking (a masked weight is an exact zero).
// On return the threads of group 0 (threadIdx.x < 128; true is returned) hold the row maxima (in log2
// units), sums and unnormalised outputs of rows RT ty .., columns 4 tx + 64 c; m = -inf, l = 0,
// o = 0 for a row that saw nothing.
template <typename T, int D, typename Shape, typename Src>
__device__ __forceinline__ bool simt_flash(const Src& src, float scale_log2e, float* smem, float (&o)[Shape::RT][D / 16],
                                           float (&m)[Shape::RT], float (&l)[Shape::RT]) {
  using S = SimtSmem<D, Shape>;
  constexpr int RT = Shape::RT, KT = Shape::KT, kRows = Shape::kRows, kKeys = Shape::kKeys;
  constexpr int ST = S::kStride, PST = S::kPStride;
  const int group = threadIdx.x / kSimtGroup, tid = threadIdx.x % kSimtGroup;
  float* sQ = smem;
  float* sK = smem + kRows * ST + group * S::kGroupFloats;
  float* sV = sK + kKeys * ST;
  float* sP = sV + kKeys * ST;
  const int tx = tid & 15, ty = tid >> 4;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o[i][c] = 0.f;
  }
  const int nt = src.n_tiles();
  auto load_k = [&](int t) {
    if (t >= nt) { cp_async_commit(); return; }   // keeps the count of pending groups
    if constexpr (Src::kGap) {
      simt_load_rows<T, D, kKeys, kSimtGroup>(sK, src.keys(t), tid, [&](int r) { return src.k(t, r); });
    } else {
      const T* base = src.k(t);
      simt_load_rows<T, D, kKeys, kSimtGroup>(sK, src.keys(t), tid, [&](int r) { return base + r * src.k_stride(); });
    }
  };
  auto load_v = [&](int t) {
    if (t >= nt) { cp_async_commit(); return; }
    if constexpr (Src::kGap) {
      simt_load_rows<T, D, kKeys, kSimtGroup>(sV, src.keys(t), tid, [&](int r) { return src.v(t, r); });
    } else {
      const T* base = src.v(t);
      simt_load_rows<T, D, kKeys, kSimtGroup>(sV, src.keys(t), tid, [&](int r) { return base + r * src.v_stride(); });
    }
  };
  __syncthreads();                         // the buffers may still be read by the item before
  simt_load_rows<T, D, kRows, kSimtThreads>(sQ, src.n_rows(), threadIdx.x, [&](int r) { return src.q(r); });
  load_k(group);
  load_v(group);
  cp_async_wait<2>();
  __syncthreads();                         // Q is shared by the groups
  for (int t = group; t < nt; t += 2) {
    cp_async_wait<1>();                    // K of this tile; V may still be on its way
    simt_group_sync(group);
    float s[RT][KT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < KT; ++j) s[i][j] = 0.f;
    auto score = [&](auto count) {         // the first count x 16 keys
      constexpr int kCount = decltype(count)::value;
#pragma unroll (RT == 4 ? 4 : 2)
      for (int d = 0; d < D; d += 4) {
        float4 q[RT], k[kCount];
#pragma unroll
        for (int i = 0; i < RT; ++i) q[i] = *reinterpret_cast<const float4*>(sQ + (ty * RT + i) * ST + d);
#pragma unroll
        for (int j = 0; j < kCount; ++j) k[j] = *reinterpret_cast<const float4*>(sK + (tx + 16 * j) * ST + d);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int j = 0; j < kCount; ++j)
            s[i][j] = fmaf(q[i].w, k[j].w, fmaf(q[i].z, k[j].z, fmaf(q[i].y, k[j].y, fmaf(q[i].x, k[j].x, s[i][j]))));
      }
    };
    if (Src::kGap && src.keys(t) <= kKeys / 2) score(std::integral_constant<int, KT / 2>{});
    else score(std::integral_constant<int, KT>{});
    simt_group_sync(group);                // K has been read
    load_k(t + 2);
    const bool masked = src.masked(t);
    int last[RT], gap0 = 0, sink0 = kKeys, n_keys = kKeys, gap1[Src::kGap ? RT : 1] = {};
    if constexpr (Src::kGap) { gap0 = src.gap_begin(t); sink0 = src.sink_begin(t); n_keys = src.keys(t); }
    auto sees = [&](int key, int last_i, int gap1_i) {
      if constexpr (Src::kGap) return key >= sink0 ? key < n_keys : key <= last_i && !(key >= gap0 && key < gap1_i);
      return key <= last_i;
    };
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      last[i] = masked ? src.last(t, ty * RT + i) : kKeys - 1;
      if constexpr (Src::kGap) gap1[i] = masked ? src.gap_end(t, ty * RT + i) : 0;
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        s[i][j] = sees(tx + 16 * j, last[i], gap1[Src::kGap ? i : 0]) ? __fmul_rn(s[i][j], scale_log2e) : -INFINITY;   // a masked score counts for nothing
        mx = fmaxf(mx, s[i][j]);
      }
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
      const float m_new = fmaxf(m[i], mx);
      const float base = (m_new == -INFINITY) ? 0.f : m_new;    // nothing seen yet: every weight is exp2(-inf) = 0
      const float corr = exp2f(m[i] - base);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        s[i][j] = exp2f(s[i][j] - base);
        sum += s[i][j];
        sP[(ty * RT + i) * PST + tx + 16 * j] = s[i][j];
      }
      l[i] = fmaf(l[i], corr, sum);        // of this thread's keys; the row's 16 threads are added up at the end
      m[i] = m_new;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[i][c] *= corr;
    }
    cp_async_wait<1>();                    // V of this tile; the next K may still be on its way
    simt_group_sync(group);                // (P needs no more than a warp: a row's 16 threads are half of one)
    auto accumulate = [&](auto guarded) {
#pragma unroll (RT == 4 ? 2 : 1)
      for (int kk = 0; kk < n_keys; kk += 4) {                       // (weights behind the tile's last key are 0)
        float4 p[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) p[i] = *reinterpret_cast<const float4*>(sP + (ty * RT + i) * PST + kk);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            const float4 v = *reinterpret_cast<const float4*>(sV + (kk + e) * ST + tx * 4 + 64 * c);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
              const float pe = e == 0 ? p[i].x : e == 1 ? p[i].y : e == 2 ? p[i].z : p[i].w;
              // a key the row does not see must not reach it even if its value is an infinity or a NaN
              if (!decltype(guarded)::value || sees(kk + e, last[i], gap1[Src::kGap ? i : 0])) {
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
    bool guard = masked;
    if constexpr (Src::kGap) {
      if (masked) {
        int top = 0;                       // of the tile's values, without their signs: from 0x7f800000 on not finite
        for (int i = tid * 4; i < kKeys * D; i += kSimtGroup * 4) {
          const int4 v = *reinterpret_cast<const int4*>(sV + i / D * ST + i % D);
          top = max(max(top, v.x & 0x7fffffff), max(v.y & 0x7fffffff, max(v.z & 0x7fffffff, v.w & 0x7fffffff)));
        }
        guard = simt_group_any(group, top >= 0x7f800000);
      }
    }
    if (guard) accumulate(std::true_type{}); else accumulate(std::false_type{});
    simt_group_sync(group);                // V has been read
    load_v(t + 2);
  }
  cp_async_wait<0>();
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
  // group 1 hands its state over through group 1's own buffers
  float* sO = smem + kRows * ST + S::kGroupFloats;
  float* sM = sO + kRows * ST;
  if (group == 1) {
    simt_group_sync(group);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        *reinterpret_cast<float4*>(sO + (ty * RT + i) * ST + tx * 4 + 64 * c) =
            make_float4(o[i][c * 4], o[i][c * 4 + 1], o[i][c * 4 + 2], o[i][c * 4 + 3]);
      if (tx == 0) {
        sM[2 * (ty * RT + i)] = m[i];
        sM[2 * (ty * RT + i) + 1] = l[i];
      }
    }
  }
  __syncthreads();
  if (group == 1) return false;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const float m1 = sM[2 * (ty * RT + i)], l1 = sM[2 * (ty * RT + i) + 1];
    const float mn = fmaxf(m[i], m1), base = (mn == -INFINITY) ? 0.f : mn;
    const float w0 = exp2f(m[i] - base), w1 = exp2f(m1 - base);
    l[i] = fmaf(l[i], w0, __fmul_rn(l1, w1));
    m[i] = mn;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      const float4 v = *reinterpret_cast<const float4*>(sO + (ty * RT + i) * ST + tx * 4 + 64 * c);
      o[i][c * 4 + 0] = fmaf(o[i][c * 4 + 0], w0, __fmul_rn(v.x, w1));
      o[i][c * 4 + 1] = fmaf(o[i][c * 4 + 1], w0, __fmul_rn(v.y, w1));
      o[i][c * 4 + 2] = fmaf(o[i][c * 4 + 2], w0, __fmul_rn(v.z, w1));
      o[i][c * 4 + 3] = fmaf(o[i][c * 4 + 3], w0, __fmul_rn(v.w, w1));
    }
  }
  return true;
}

}  // namespace tca
