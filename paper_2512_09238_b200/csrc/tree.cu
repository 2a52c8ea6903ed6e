// tca_attn_tree: attention of a tree of drafted tokens over the retained cache (Eq. 2 for several query
// tokens at once, speculative decoding).  Query (head, t) sees every row of its unit's cache and the
// drafted tokens on its own path to the root.
//
// Two parts.  The cache is the same for all G * T query rows of a unit, so its rows are cut into slices
// and a split kernel attends a block of query rows to one slice (this file: FP32 pipes; tree_tc.cu: tensor
// cores).  The drafted part is a walk, no product of matrices: the combine kernel, one warp per query row, walks
// the path to the root, attends to exactly the tokens on it (a drafted token outside the path is not read,
// whatever it holds) and merges the partial results of the cache in order.  That suits trees whose paths are short.
// It costs path length times rows, and the rows of a group and of a common prefix share nothing: a chain of 32
// tokens over 600 cached ones takes 26 us, of 128 101 us, where as many separate roots take 13 and 19 us (32 heads
// of 128).  The merge is a chain of dependent loads: 5 to 6 us after the split kernel's end, for 2048 rows of 9 to
// 19 partial results each (up to 19 MB, from L2).  One KV head alone has 296 results per row (41K cached
// tokens, 4 drafted: 60 us, with eight KV heads 38 us).
#include "flash_simt.cuh"
#include "tree_common.cuh"

namespace tca {

int launch_tree_tc(const tca_params* prm, const void* q, const tca_cache_desc* c, const TreePlan& plan, const TreeWs& ws,
                   cudaStream_t s);

namespace {
bool tree_on_tensor_cores(const tca_params* prm) { return prm->dtype == TCA_BF16 && !(prm->flags & TCA_FLAG_PREFILL_SIMT); }
}  // namespace

TreePlan tree_plan(const tca_params* prm, int n_draft) {
  TreePlan p;
  const int U = prm->batch * prm->n_kv_heads;
  const bool tc = tree_on_tensor_cores(prm);
  p.rows = prm->n_q_heads / prm->n_kv_heads * n_draft;
  // tensor cores: up to 128 rows run as two streams over alternate tiles, more as two blocks per CTA
  p.streams = tc && p.rows <= 128 ? 2 : 1;
  p.rows_per_cta = !tc ? SimtSmall::kRows : p.rows <= 128 ? 128 : 256;
  p.row_blocks = (p.rows + p.rows_per_cta - 1) / p.rows_per_cta;
  p.min_share = tc ? 2 : 1;
  p.lead = tc ? 3 : 0;
  const int resident = (tc ? 1 : prm->head_dim == 128 ? SimtSmem<128, SimtSmall>::kCtasPerSm : SimtSmem<64, SimtSmall>::kCtasPerSm) * sm_count();
  p.n_shares = resident / p.row_blocks > 0 ? resident / p.row_blocks : 1;
  p.n_slots = p.n_shares + U;
  return p;
}

namespace {

template <typename T, int D>
struct TreeSrc {
  const T *q_rows, *Kc, *Vc;      // first query row of this CTA; the cache
  int n;                          // query rows here
  SliceTiles<SimtSmall::kKeys> tiles;
  __device__ __forceinline__ int n_rows() const { return n; }
  __device__ __forceinline__ int n_tiles() const { return tiles.n_tiles(); }
  __device__ __forceinline__ int keys(int t) const { int y, c; tiles.get(t, y, c); return c; }
  __device__ __forceinline__ const T* q(int r) const { return q_rows + int64_t(r) * D; }
  __device__ __forceinline__ const T* k(int t) const { int y, c; tiles.get(t, y, c); return Kc + int64_t(y) * D; }
  __device__ __forceinline__ const T* v(int t) const { int y, c; tiles.get(t, y, c); return Vc + int64_t(y) * D; }
  __device__ __forceinline__ int k_stride() const { return D; }
  __device__ __forceinline__ int v_stride() const { return D; }
  __device__ __forceinline__ bool masked(int t) const { return keys(t) < SimtSmall::kKeys; }
  __device__ __forceinline__ int last(int t, int) const { return keys(t) - 1; }
};

template <typename T, int D>
__global__ void __launch_bounds__(kSimtThreads, SimtSmem<D, SimtSmall>::kCtasPerSm)
tree_simt_kernel(const T* __restrict__ q, const T* __restrict__ Kc, const T* __restrict__ Vc,
                 const int64_t* __restrict__ state, int n_units, int64_t tail_cap, TreePlan plan, float scale_log2e,
                 TreeWs ws) {
  extern __shared__ float4 tree_smem[];
  __shared__ TreePiece<SimtSmall::kKeys> piece;
  pdl_wait();
  pdl_launch_dependents();
  const int share = int(blockIdx.x) / plan.row_blocks, rb = int(blockIdx.x) % plan.row_blocks;
  const int row0 = rb * SimtSmall::kRows;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;   // of the group that writes
  TreeFinder finder;
  if (threadIdx.x < 32) finder.start(state, n_units, plan, share, threadIdx.x);
  for (;;) {
    if (threadIdx.x < 32) {
      TreePiece<SimtSmall::kKeys> p;
      const bool more = finder.next(state, n_units, int(tail_cap), share, rb == 0, ws.table, threadIdx.x, p);
      if (!more) p.u = -1;
      if (threadIdx.x == 0) piece = p;
    }
    __syncthreads();
    const TreePiece<SimtSmall::kKeys> mine = piece;
    __syncthreads();                       // read by all before the next one is written
    if (mine.u < 0) return;
    TreeSrc<T, D> src;
    src.n = min(SimtSmall::kRows, plan.rows - row0);
    src.q_rows = q + (int64_t(mine.u) * plan.rows + row0) * D;
    src.Kc = Kc;
    src.Vc = Vc;
    src.tiles = mine.tiles;
    float o[4][D / 16], m[4], l[4];
    const bool mine_to_write = simt_flash<T, D, SimtSmall>(src, scale_log2e, reinterpret_cast<float*>(tree_smem), o, m, l);
#pragma unroll
    for (int i = 0; i < 4 && mine_to_write; ++i) {
      const int r = row0 + ty * 4 + i;
      if (r >= plan.rows) continue;
      const size_t at = size_t(mine.slot) * plan.rows + r;
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        *reinterpret_cast<float4*>(ws.acc + at * D + tx * 4 + 64 * c) =
            make_float4(o[i][c * 4], o[i][c * 4 + 1], o[i][c * 4 + 2], o[i][c * 4 + 3]);
      if (tx == 0) ws.ml[at] = make_float2(m[i], l[i]);
    }
  }
}

// ------------------------------------------------------------------ drafted tokens, and the merge of the slices
constexpr int kCombineWarps = 8;

template <int E>
struct RowE {   // E = D / 32 consecutive elements per lane
  float x[E];
  __device__ __forceinline__ void load(const float* p) {
    if constexpr (E == 4) { const float4 v = *reinterpret_cast<const float4*>(p); x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
    else { const float2 v = *reinterpret_cast<const float2*>(p); x[0] = v.x; x[1] = v.y; }
  }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    if constexpr (E == 4) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
    } else {
      const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
      x[0] = bf16_lo(v); x[1] = bf16_hi(v);
    }
  }
  __device__ __forceinline__ void store(float* p) const {
    if constexpr (E == 4) *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    else *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]);
  }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const {
#pragma unroll
    for (int e = 0; e < E; e += 2)
      *reinterpret_cast<__nv_bfloat162*>(p + e) = __floats2bfloat162_rn(x[e], x[e + 1]);
  }
};

// One warp per query row.  The drafted part comes before the dependency wait: it reads the caller's inputs
// only, which were complete before the split kernel could start (that kernel triggers this launch after its
// own wait).  It overlaps the split kernel where that leaves room: a CTA of the tensor-core kernel fills its SM, so
// only CTAs that find an SM already left run ahead, and a long walk adds to the call.  Every loop issues its loads ahead of the arithmetic that
// depends on them: with one row per warp the kernel is bound by latency.
template <typename T, int D>
__global__ void __launch_bounds__(kCombineWarps * 32)
tree_combine_kernel(const T* __restrict__ q, const T* __restrict__ k_draft, const T* __restrict__ v_draft, int n_draft,
                    const int32_t* __restrict__ parent, const int32_t* __restrict__ n_live,
                    const int64_t* __restrict__ state, int n_kv, TreePlan plan, float scale_log2e, TreeWs ws,
                    T* __restrict__ O) {
  constexpr int E = D / 32;
  constexpr int kHeld = TCA_TREE_MAX / 32;
  constexpr int kBatch = 4;        // drafted tokens whose rows are fetched together
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = blockIdx.x * kCombineWarps + warp, u = blockIdx.y, seq = u / n_kv;
  const int t = r % n_draft;
  // not a row, or not drafted: its row of O stays as it was
  const bool live = r < plan.rows && (!n_live || t < n_live[seq]);
  RowE<E> o, qr;
#pragma unroll
  for (int e = 0; e < E; ++e) o.x[e] = 0.f;
  float m = -INFINITY, l = 0.f;
  const size_t q_at = (size_t(u) * plan.rows + r) * D + lane * E;
  int64_t cached = 0;
  if (live) {
    const int64_t* st = state + size_t(u) * TCA_STATE_WORDS;
    cached = st[TCA_ST_N_GLOBAL] + st[TCA_ST_N_TAIL];
    qr.load(q + q_at);
    // the path to the root as a bit set: parents lie in the lanes, a hop is one shuffle
    int par[kHeld];
    unsigned bits[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      par[i] = i * 32 + lane < n_draft ? parent[size_t(seq) * n_draft + i * 32 + lane] : -1;
      bits[i] = 0;
    }
    for (int cur = t; cur >= 0;) {
      int p = -1;
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (i == (cur >> 5)) {
          bits[i] |= 1u << (cur & 31);
          p = par[i];
        }
      p = __shfl_sync(0xffffffffu, p, cur & 31);
      if constexpr (kDebugBounds) {
        if (lane == 0 && (p < -1 || p >= cur)) report_bounds_ws(ws.status, kBoundsDraftIndex, p);
      }
      cur = p < cur ? p : -1;                                // a parent that does not precede its child ends the path
    }
    const T* kd = k_draft + size_t(u) * n_draft * D + lane * E;
    const T* vd = v_draft + size_t(u) * n_draft * D + lane * E;
    bool more = true;
    while (more) {
      int a[kBatch];
      RowE<E> k[kBatch], v[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        a[b] = -1;
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
          if (a[b] < 0 && bits[i]) {
            a[b] = i * 32 + __ffs(bits[i]) - 1;
            bits[i] &= bits[i] - 1;
          }
        if (a[b] >= 0) {
          k[b].load(kd + size_t(a[b]) * D);
          v[b].load(vd + size_t(a[b]) * D);
        }
      }
      more = a[kBatch - 1] >= 0;
      float x[kBatch], mn = m;
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        x[b] = -INFINITY;
        if (a[b] < 0) continue;                              // uniform
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s = fmaf(qr.x[e], k[b].x[e], s);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        x[b] = s * scale_log2e;
        mn = fmaxf(mn, x[b]);
      }
      const float base = (mn == -INFINITY) ? 0.f : mn, c = exp2f(m - base);
      l *= c;
#pragma unroll
      for (int e = 0; e < E; ++e) o.x[e] *= c;
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        if (a[b] < 0) continue;
        const float w = exp2f(x[b] - base);
        l += w;
#pragma unroll
        for (int e = 0; e < E; ++e) o.x[e] = fmaf(w, v[b].x[e], o.x[e]);
      }
      m = mn;
    }
  }
  pdl_wait();                 // the partial results come from the split kernel
  pdl_launch_dependents();
  if (!live) return;
  // the unit's partial results, in the order of its rows; a unit whose cache is empty has none.  (Both words
  // are requested before either is looked at.)
  const int2 where = cached > 0 ? __ldcg(ws.table + u) : make_int2(0, 0);
  if (stops_call(__ldcg(ws.status))) return;      // a wait gave up: there are no partial results
  const int n = min(where.y, plan.n_slots - where.x) * plan.streams;
  const size_t first = size_t(where.x) * plan.streams;
  for (int c0 = 0; c0 < n; c0 += 32) {                       // statistics of 32 partials at a time, one per lane
    const int cn = min(32, n - c0);
    const float2 ml = lane < cn ? ws.ml[(first + c0 + lane) * plan.rows + r] : make_float2(-INFINITY, 0.f);
    float mn = ml.x;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, off));
    mn = fmaxf(m, mn);
    const float base = (mn == -INFINITY) ? 0.f : mn, keep = exp2f(m - base);
    // a stream without a tile wrote no output (maximum -inf, sum 0); one whose scores are all NaN has no maximum
    // either, but a sum that is NaN and has to reach the result
    const bool some = ml.x != -INFINITY || ml.y != 0.f;
    const float w = some ? exp2f(ml.x - base) : 0.f;
    const unsigned have = __ballot_sync(0xffffffffu, some);
    l *= keep;
#pragma unroll
    for (int e = 0; e < E; ++e) o.x[e] *= keep;
    const float wl = some ? w * ml.y : 0.f;
#pragma unroll 8
    for (int c = 0; c < cn; ++c) {
      const float wc = __shfl_sync(0xffffffffu, w, c);
      l += __shfl_sync(0xffffffffu, wl, c);
      if (!((have >> c) & 1u)) continue;                     // uniform
      RowE<E> a;
      a.load(ws.acc + ((first + c0 + c) * plan.rows + r) * D + lane * E);
#pragma unroll
      for (int e = 0; e < E; ++e) o.x[e] = fmaf(wc, a.x[e], o.x[e]);
    }
    m = mn;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) o.x[e] /= l;
  o.store(O + q_at);
}

template <typename T, int D>
int launch_tree(const tca_params* prm, const void* q, const void* kd, const void* vd, int n_draft, const int32_t* parent,
                const int32_t* n_live, const tca_cache_desc* c, void* O, const TreePlan& plan, const TreeWs& ws,
                cudaStream_t s) {
  const int U = prm->batch * prm->n_kv_heads;
  const float scale = prm->sm_scale * 1.4426950408889634f;
  const int64_t ctas = int64_t(plan.n_shares) * plan.row_blocks;
  if (ctas >= (int64_t(1) << 31)) return TCA_ERR_UNSUPPORTED;
  int st;
  if (tree_on_tensor_cores(prm)) {
    st = launch_tree_tc(prm, q, c, plan, ws, s);
  } else {
    auto kern = tree_simt_kernel<T, D>;
    if (allow_smem<tree_simt_kernel<T, D>>(SimtSmem<D, SimtSmall>::kBytes) != TCA_OK) return TCA_ERR_CUDA;
    st = launch_pdl(kern, dim3(unsigned(ctas)), dim3(kSimtThreads), size_t(SimtSmem<D, SimtSmall>::kBytes), s,
                    static_cast<const T*>(q), static_cast<const T*>(c->k), static_cast<const T*>(c->v),
                    static_cast<const int64_t*>(c->state), U, c->tail_cap, plan, scale, ws);
  }
  if (st != TCA_OK) return st;
  return launch_pdl(tree_combine_kernel<T, D>, dim3(unsigned((plan.rows + kCombineWarps - 1) / kCombineWarps), unsigned(U)),
                    dim3(kCombineWarps * 32), size_t(0), s, static_cast<const T*>(q), static_cast<const T*>(kd),
                    static_cast<const T*>(vd), n_draft, parent, n_live, static_cast<const int64_t*>(c->state),
                    prm->n_kv_heads, plan, scale, ws, static_cast<T*>(O));
}

bool bad_tree_shape(const tca_params* prm, int32_t n_draft) {
  return n_draft > TCA_TREE_MAX || int64_t(prm->batch) * prm->n_kv_heads > 65535;
}

}  // namespace
}  // namespace tca

using namespace tca;

extern "C" size_t tca_attn_tree_workspace_bytes(const tca_params* prm, int32_t n_draft) {
  if (check_params(prm) != TCA_OK || n_draft < 1 || bad_tree_shape(prm, n_draft)) return 0;
  size_t most = 0;   // fewer rows can need more (they run as two streams): one workspace serves all calls up to n_draft
  for (int32_t n = 1; n <= n_draft; ++n) {
    const size_t bytes = tree_ws_layout(prm, tree_plan(prm, n), nullptr).bytes;
    most = bytes > most ? bytes : most;
  }
  return most;
}

extern "C" int tca_attn_tree(const tca_params* prm, const void* q, const void* k_draft, const void* v_draft,
                             int32_t n_draft, const int32_t* parent, const int32_t* n_live, const tca_cache_desc* c,
                             void* O, void* ws, size_t ws_bytes, void* stream) {
  int st = check_params(prm);
  if (st != TCA_OK) return st;
  TCA_CHECK_ARG(q && k_draft && v_draft && parent && c && O && ws && n_draft >= 1);
  TCA_CHECK_ARG(c->k && c->v && c->state);
  TCA_CHECK_ARG(aligned(q, 16) && aligned(k_draft, 16) && aligned(v_draft, 16) && aligned(O, 16) && aligned(ws, 256));
  TCA_CHECK_ARG(aligned(c->k, 16) && aligned(c->v, 16) && aligned(parent, 4) && aligned(n_live, 4));
  TCA_CHECK_ARG(c->n_units == int64_t(prm->batch) * prm->n_kv_heads && c->tail_cap >= 1);
  TCA_CHECK_ARG(c->rows_total >= 1 && c->rows_total < (int64_t(1) << 31));
  if (bad_tree_shape(prm, n_draft)) return TCA_ERR_UNSUPPORTED;
  const TreePlan plan = tree_plan(prm, n_draft);
  const TreeWs lay = tree_ws_layout(prm, plan, ws);
  if (ws_bytes < lay.bytes) return TCA_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
#define TCA_TREE(T, D) launch_tree<T, D>(prm, q, k_draft, v_draft, n_draft, parent, n_live, c, O, plan, lay, s)
  if (prm->dtype == TCA_F32) return prm->head_dim == 128 ? TCA_TREE(float, 128) : TCA_TREE(float, 64);
  return prm->head_dim == 128 ? TCA_TREE(__nv_bfloat16, 128) : TCA_TREE(__nv_bfloat16, 64);
#undef TCA_TREE
}
