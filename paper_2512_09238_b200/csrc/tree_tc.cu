// The cache part of tca_attn_tree for bf16, on the tensor cores: a block of up to 256 query rows (G heads
// x drafted tokens) against one slice of a unit's cache rows.  Bound by memory while the rows are few
// (every cache row is read once per 256 query rows), by the tensor pipe and the exponentials from about
// 128 rows on.
#include "flash_tc.cuh"
#include "tree_common.cuh"

namespace tca {
namespace {

template <int D, bool kShared>
struct TreeTcSrc {
  const CUtensorMap *mq, *mk, *mv;
  SliceTiles slice;
  int q_row;        // first query row of this CTA in the flattened query matrix
  int rows;         // query rows of this CTA
  int n;            // tiles of the slice
  float* acc;       // partial results: first row of this CTA in the first stream's block
  float2* ml;
  size_t stream_stride;   // rows from one stream's block to the next

  __device__ __forceinline__ int tiles(int h) const { return kShared && h * kTcRows >= rows ? 0 : n; }
  __device__ __forceinline__ int q_bytes(int) const { return TcLayout<D>::kTile; }
  __device__ __forceinline__ void load_q(int h, uint8_t* dst, uint64_t* bar) const {
    for (int half = 0; half < D / 64; ++half)
      ptx::tma_load_2d(dst + half * kTcHalfBytes, mq, half * 64, q_row + h * kTcRows, bar);
  }
  __device__ __forceinline__ void load(int t, bool is_v, uint8_t* dst, uint64_t* bar) const {
    int y, c;
    slice.get(t, y, c);
    for (int half = 0; half < D / 64; ++half)
      ptx::tma_load_2d(dst + half * kTcHalfBytes, is_v ? mv : mk, half * 64, y, bar);
  }
  __device__ __forceinline__ int row_key(int, int) const { return 0; }
  __device__ __forceinline__ int last(int, int t) const {
    int y, c;
    slice.get(t, y, c);
    return c - 1;
  }
  // rows behind a run's end are another unit's or not in use
  __device__ __forceinline__ int clean(int t) const {
    int y, c;
    slice.get(t, y, c);
    return c < kTcKeys ? c : -1;
  }
  __device__ __forceinline__ bool scan() const { return false; }
  __device__ __forceinline__ int note_slot(int) const { return 0; }

  template <typename Read>
  __device__ __forceinline__ void store(int h, int row, bool seen, float m, float l, Read read) const {
    const int r = kShared ? h * kTcRows + row : row;
    const size_t at = (kShared ? 0 : size_t(h) * stream_stride) + r;
    if (r < rows) ml[at] = seen ? make_float2(m, l) : make_float2(-INFINITY, 0.f);
    if (!seen) return;
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t v[32];
      read(c, v);
      if (r < rows) {
#pragma unroll
        for (int k = 0; k < 32; k += 4)
          *reinterpret_cast<uint4*>(acc + at * D + c * 32 + k) = make_uint4(v[k], v[k + 1], v[k + 2], v[k + 3]);
      }
    }
  }
};

template <int D, bool kShared>
__global__ void __launch_bounds__(kTcThreads, 1)
tree_tc_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
               const __grid_constant__ CUtensorMap mv, const int64_t* __restrict__ state, int n_units, int64_t tail_cap,
               TreePlan plan, float scale_log2e, TreeWs ws) {
  extern __shared__ uint8_t tree_tc_smem[];
  __shared__ TcShared sh;
  __shared__ TreeSlice slice;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(tree_tc_smem) + 1023) & ~uintptr_t(1023));
  if (threadIdx.x == 0) {
    ptx::tma_prefetch_desc(&mq);
    ptx::tma_prefetch_desc(&mk);
    ptx::tma_prefetch_desc(&mv);
  }
  pdl_wait();
  pdl_launch_dependents();
  if (threadIdx.x < 32) {
    const TreeSlice s = tree_find(state, n_units, tail_cap, plan.n_slots, plan.step_rows, plan.min_steps, kTcKeys,
                                  int(blockIdx.x) / plan.row_blocks, threadIdx.x);
    if (threadIdx.x == 0) slice = s;
  }
  __syncthreads();
  if (slice.u < 0) return;
  const int rb = int(blockIdx.x) % plan.row_blocks;
  if (slice.part == 0 && rb == 0 && threadIdx.x == 0) ws.table[slice.u] = make_int2(slice.base, slice.np);
  TreeTcSrc<D, kShared> src;
  src.mq = &mq; src.mk = &mk; src.mv = &mv;
  src.slice = slice.tiles;
  src.n = src.slice.n_tiles();
  const int row0 = rb * plan.rows_per_cta;
  src.q_row = slice.u * plan.rows + row0;
  src.rows = min(plan.rows_per_cta, plan.rows - row0);
  const size_t at = size_t(slice.base + slice.part) * plan.streams * plan.rows + row0;
  src.acc = ws.acc + at * D;
  src.ml = ws.ml + at;
  src.stream_stride = size_t(plan.rows);
  flash_tc<D, kShared>(src, smem, &sh, scale_log2e, ws.status);
}

template <int D, bool kShared>
int launch(const tca_params* prm, const void* q, const tca_cache_desc* c, const TreePlan& plan, const TreeWs& ws,
           cudaStream_t s) {
  const int U = prm->batch * prm->n_kv_heads;
  CUtensorMap mq, mk, mv;
  if (!encode_map(&mq, q, D, int64_t(U) * plan.rows, 0, 0) || !encode_map(&mk, c->k, D, c->rows_total, 0, 0) ||
      !encode_map(&mv, c->v, D, c->rows_total, 0, 0))
    return TCA_ERR_CUDA;
  auto kern = tree_tc_kernel<D, kShared>;
  TCA_CHECK_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, TcLayout<D>::bytes));
  return launch_pdl(kern, dim3(unsigned(plan.n_slots * plan.row_blocks)), dim3(kTcThreads), size_t(TcLayout<D>::bytes), s, mq,
                    mk, mv, static_cast<const int64_t*>(c->state), U, c->tail_cap, plan,
                    prm->sm_scale * 1.4426950408889634f, ws);
}

}  // namespace

int launch_tree_tc(const tca_params* prm, const void* q, const tca_cache_desc* c, const TreePlan& plan, const TreeWs& ws,
                   cudaStream_t s) {
  const bool shared = plan.streams == 1;
  if (prm->head_dim == 128)
    return shared ? launch<128, true>(prm, q, c, plan, ws, s) : launch<128, false>(prm, q, c, plan, ws, s);
  return shared ? launch<64, true>(prm, q, c, plan, ws, s) : launch<64, false>(prm, q, c, plan, ws, s);
}

}  // namespace tca
