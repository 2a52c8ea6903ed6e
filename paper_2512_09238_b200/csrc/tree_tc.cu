// The cache part of tca_attn_tree for bf16, on the tensor cores: a block of up to 256 query rows (G heads
// x drafted tokens) against the pieces of a share of the cache rows.  Bound by memory while the rows are few
// (every cache row is read once per 256 query rows), by the tensor pipe and the exponentials from about
// 128 rows on.  206 MB of cache for 4 x 16 drafted tokens (64 rows per unit): 33 us of streaming at
// 6.2 TB/s after a start of 5 us; 155 MB for 64 drafted tokens (256 rows): 38 us, 1.0 PFLOP/s.
#include "flash_tc.cuh"
#include "tree_common.cuh"

namespace tca {
namespace {

struct TreeItem {
  SliceTiles<kTcKeys> slice;
  int q_row;        // first query row of this CTA in the flattened query matrix
  size_t at;        // partial results: its first row in the first stream's block
};

// The items of a CTA: its block of query rows against the pieces of its share, one after the other.
template <int D, bool kShared>
struct TreeTcSrc {
  using Item = TreeItem;
  const CUtensorMap *mq, *mk, *mv;
  const int64_t* state;
  int n_units;
  int tail_cap;
  const TreePlan* plan;
  uint64_t stream;      // the cache streams through the L2: its lines go first
  const TreeWs* ws;
  int share, rb, rows;  // rows: query rows of this CTA
  SliceTiles<kTcKeys> slice;
  int q_row, n;
  size_t at0;
  TreeFinder finder;    // the producer warp's

  __device__ __forceinline__ void begin(int lane) { finder.start(state, n_units, *plan, share, lane); }
  __device__ __forceinline__ bool find(int, int lane, Item& it) {
    TreePiece<kTcKeys> p;
    if (!finder.next(state, n_units, tail_cap, share, rb == 0, ws->table, lane, p)) return false;
    const int row0 = rb * plan->rows_per_cta;
    it.slice = p.tiles;
    it.q_row = p.u * plan->rows + row0;
    it.at = size_t(p.slot) * plan->streams * plan->rows + row0;
    return true;
  }
  __device__ __forceinline__ void set(const Item& it) {
    slice = it.slice; q_row = it.q_row; at0 = it.at;
    n = slice.n_tiles();
  }
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
      ptx::tma_load_2d_hint(dst + half * kTcHalfBytes, is_v ? mv : mk, half * 64, y, bar, stream);
  }
  int row;
  __device__ __forceinline__ void begin_row(int r) { row = r; }
  __device__ __forceinline__ int row_key(int) const { return 0; }
  __device__ __forceinline__ int last(int, int t) const {
    int y, c;
    slice.get(t, y, c);
    return c - 1;
  }
  __device__ __forceinline__ int keys(int, int t) const {
    int y, c;
    slice.get(t, y, c);
    return c;
  }
  __device__ __forceinline__ int whole_tiles() const { return slice.n_whole(); }
  // rows behind a run's end are another unit's or not in use
  __device__ __forceinline__ int clean(int t) const {
    int y, c;
    slice.get(t, y, c);
    return c < kTcKeys ? c : -1;
  }
  __device__ __forceinline__ int scan_from(int) const { return kTcKeys; }
  __device__ __forceinline__ int note_slot(int) const { return 0; }

  template <typename Read>
  __device__ __forceinline__ void store(int h, bool seen, float m, float l, const uint32_t*, Read read) const {
    const int r = kShared ? h * kTcRows + row : row;
    const size_t at = at0 + (kShared ? 0 : size_t(h) * plan->rows) + r;
    if (r < rows) ws->ml[at] = seen ? make_float2(m, l) : make_float2(-INFINITY, 0.f);
    if (!seen) return;
    const TcRowOut rows_out(r < rows ? ws->acc + at * D : nullptr);
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t v[32];
      read(c, v);
      ptx::tc_wait_ld();
      rows_out.store32(v, c * 128);
    }
  }
};

template <int D, bool kShared>
__global__ void __launch_bounds__(kTcThreads, 1)
tree_tc_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
               const __grid_constant__ CUtensorMap mv, const int64_t* __restrict__ state, int n_units, int64_t tail_cap,
               const __grid_constant__ TreePlan plan, float scale_log2e, const __grid_constant__ TreeWs ws) {
  extern __shared__ uint8_t tree_tc_smem[];
  __shared__ TcShared<TreeItem> sh;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(tree_tc_smem) + 1023) & ~uintptr_t(1023));
  if (threadIdx.x == 0) {
    ptx::tma_prefetch_desc(&mq);
    ptx::tma_prefetch_desc(&mk);
    ptx::tma_prefetch_desc(&mv);
  }
  flash_tc_setup<D>(smem, &sh);
  pdl_wait();
  pdl_launch_dependents();
  TreeTcSrc<D, kShared> src;
  src.mq = &mq; src.mk = &mk; src.mv = &mv;
  src.state = state;
  src.n_units = n_units;
  src.tail_cap = int(tail_cap);
  src.stream = ptx::l2_policy_evict_first();
  src.plan = &plan;
  src.ws = &ws;
  src.share = int(blockIdx.x) / plan.row_blocks;
  src.rb = int(blockIdx.x) % plan.row_blocks;
  src.rows = min(plan.rows_per_cta, plan.rows - src.rb * plan.rows_per_cta);
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
  if (allow_smem<tree_tc_kernel<D, kShared>>(TcLayout<D>::bytes) != TCA_OK) return TCA_ERR_CUDA;
  return launch_pdl(kern, dim3(unsigned(plan.n_shares * plan.row_blocks)), dim3(kTcThreads), size_t(TcLayout<D>::bytes), s, mq,
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
