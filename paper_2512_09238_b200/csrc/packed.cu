// tca_attn_packed: causal attention of prompts of different lengths packed one after another (Eq. 2
// with every key retained), grouped query heads, strided buffers.  This file holds the entry point and
// the FP32-pipe kernel (fp32 inputs; bf16 with TCA_FLAG_PREFILL_SIMT as a cross-check); bf16 runs on
// the tensor-core kernel of packed_tc.cu.
#include "flash_simt.cuh"
#include "packed_common.cuh"

namespace tca {

template <int D>
int launch_packed_tc(const tca_params* prm, const void* Q, const void* K, const void* V, const PackedArgs& a, void* O,
                     void* ws, cudaStream_t s);

namespace {

// Query rows of a CTA are (position, head of the group) pairs, head fastest: row r is position
// p0 + r / G, head kvh * G + r % G, so a short sequence of a wide group still fills the tile.
template <typename T, typename Shape>
struct PackedSrc {
  static constexpr int kRows = Shape::kRows, kKeys = Shape::kKeys;
  const T *Q, *K, *V;
  const PackedArgs* a;
  PackedWork w;
  int G;
  __device__ __forceinline__ int n_rows() const { return min(kRows / G, w.len - w.p0) * G; }
  __device__ __forceinline__ int last_pos() const { return w.p0 + n_rows() / G - 1; }
  __device__ __forceinline__ int n_tiles() const { return last_pos() / kKeys + 1; }
  __device__ __forceinline__ int keys(int t) const { return min(kKeys, last_pos() + 1 - t * kKeys); }
  __device__ __forceinline__ const T* q(int r) const {
    return Q + (w.kvh * G + r % G) * a->q.head + (w.row0 + w.p0 + r / G) * a->q.row;
  }
  __device__ __forceinline__ const T* k(int t) const { return K + w.kvh * a->k.head + (w.row0 + t * kKeys) * a->k.row; }
  __device__ __forceinline__ const T* v(int t) const { return V + w.kvh * a->v.head + (w.row0 + t * kKeys) * a->v.row; }
  __device__ __forceinline__ int64_t k_stride() const { return a->k.row; }
  __device__ __forceinline__ int64_t v_stride() const { return a->v.row; }
  __device__ __forceinline__ bool masked(int t) const { return (t + 1) * kKeys - 1 > w.p0; }
  __device__ __forceinline__ int last(int t, int r) const { return min(w.p0 + r / G, last_pos()) - t * kKeys; }
};

template <typename T, int D, typename Shape>
__global__ void __launch_bounds__(kSimtThreads, SimtSmem<D, Shape>::kCtasPerSm)
packed_simt_kernel(const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const __grid_constant__ PackedArgs args,
                   float scale_log2e, T* __restrict__ O) {
  extern __shared__ float4 packed_smem[];
  __shared__ PackedWork found;
  __shared__ int held[PackedFinder::kHeld];
  pdl_wait();
  pdl_launch_dependents();
  const int G = args.n_q_heads / args.n_kv_heads;
  const int tile_pos = Shape::kRows / G;
  PackedSrc<T, Shape> src;
  src.Q = Q; src.K = K; src.V = V; src.a = &args; src.G = G;
  if (threadIdx.x < 32) {
    PackedFinder finder;
    finder.read(args, tile_pos, threadIdx.x, held);
    PackedWork w;
    int tile = 0;
    w.len = 0;
    if (finder.find(args, int(blockIdx.x) / args.n_kv_heads, tile_pos, threadIdx.x, w.row0, w.len, tile)) {
      w.p0 = tile * tile_pos;
      w.kvh = int(blockIdx.x) % args.n_kv_heads;
    }
    if (threadIdx.x == 0) found = w;
  }
  __syncthreads();
  src.w = found;
  if (src.w.len == 0) return;
  constexpr int RT = Shape::RT;
  float o[RT][D / 16], m[RT], l[RT];
  if (!simt_flash<T, D, Shape>(src, scale_log2e, reinterpret_cast<float*>(packed_smem), o, m, l)) return;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int r = ty * RT + i;
    if (r >= src.n_rows()) continue;
    T* out = O + (src.w.kvh * G + r % G) * args.o.head + (src.w.row0 + src.w.p0 + r / G) * args.o.row;
    const float inv = 1.f / l[i];
#pragma unroll
    for (int c = 0; c < D / 16; ++c) store_elt(out + tx * 4 + 64 * (c / 4) + c % 4, o[i][c] * inv);
  }
}

template <typename T, int D, typename Shape>
int launch_packed_shape(const tca_params* prm, const void* Q, const void* K, const void* V, const PackedArgs& a, void* O,
                        cudaStream_t s) {
  using Smem = SimtSmem<D, Shape>;
  const int64_t n = packed_max_tiles(a.rows, a.n_seq, Shape::kRows / (a.n_q_heads / a.n_kv_heads)) * a.n_kv_heads;
  if (n >= (int64_t(1) << 31)) return TCA_ERR_UNSUPPORTED;
  constexpr auto kern = packed_simt_kernel<T, D, Shape>;
  if (allow_smem<kern>(Smem::kBytes) != TCA_OK) return TCA_ERR_CUDA;
  return launch_pdl(kern, dim3(unsigned(n)), dim3(kSimtThreads), size_t(Smem::kBytes), s, static_cast<const T*>(Q),
                    static_cast<const T*>(K), static_cast<const T*>(V), a, prm->sm_scale * 1.4426950408889634f,
                    static_cast<T*>(O));
}

// The large tiles where they give every SM more than one CTA and are not mostly padding: prompts that
// average four of them.
template <typename T, int D>
int launch_packed_simt(const tca_params* prm, const void* Q, const void* K, const void* V, const PackedArgs& a, void* O,
                       cudaStream_t s) {
  using Large = SimtLarge;
  const int64_t tiles = a.rows * a.n_q_heads / Large::kRows;
  if (tiles >= sm_count() && a.rows * (a.n_q_heads / a.n_kv_heads) >= int64_t(4) * Large::kRows * a.n_seq)
    return launch_packed_shape<T, D, Large>(prm, Q, K, V, a, O, s);
  return launch_packed_shape<T, D, SimtSmall>(prm, Q, K, V, a, O, s);
}

// A buffer's strides: multiples of 16 bytes (vector loads, tensor maps), and room for a row.
bool bad_view(const PackedView& v, const tca_params* prm) {
  const int64_t unit = 16 / int64_t(elt_size(prm->dtype));
  constexpr int64_t kMost = int64_t(1) << 36;   // elements: below the 2^40-byte limit of a tensor map's stride
  return v.head < prm->head_dim || v.row < prm->head_dim || v.head % unit || v.row % unit || v.head >= kMost || v.row >= kMost;
}

}  // namespace
}  // namespace tca

using namespace tca;

extern "C" int tca_attn_packed(const tca_params* prm, const void* Q, const void* K, const void* V, int64_t rows,
                               const int64_t* seq_start, const int64_t* strides, void* O, void* ws, size_t ws_bytes,
                               void* stream) {
  int st = check_params(prm);
  if (st != TCA_OK) return st;
  TCA_CHECK_ARG(((Q && K && V && O) || rows == 0) && seq_start && ws);   // no rows: nothing that they would point at
  TCA_CHECK_ARG(rows >= 0 && rows < (int64_t(1) << 31));
  TCA_CHECK_ARG(aligned(Q, 16) && aligned(K, 16) && aligned(V, 16) && aligned(O, 16) && aligned(ws, 256));
  TCA_CHECK_ARG(aligned(seq_start, 8));
  PackedArgs a;
  PackedView* views[4] = {&a.q, &a.k, &a.v, &a.o};
  for (int i = 0; i < 4; ++i) {
    *views[i] = strides ? PackedView{strides[2 * i], strides[2 * i + 1]}
                        : PackedView{(rows > 0 ? rows : 1) * prm->head_dim, int64_t(prm->head_dim)};
    TCA_CHECK_ARG(!bad_view(*views[i], prm));
  }
  if (ws_bytes < tca_workspace_bytes(prm, rows > 0 ? rows : 1, TCA_OP_PACKED)) return TCA_ERR_WORKSPACE;
  if (rows == 0) return TCA_OK;   // nothing to compute
  a.rows = rows;
  a.seq_start = seq_start;
  a.n_seq = prm->batch;
  a.n_q_heads = prm->n_q_heads;
  a.n_kv_heads = prm->n_kv_heads;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (prm->dtype == TCA_F32) {
    if (prm->head_dim == 128) return launch_packed_simt<float, 128>(prm, Q, K, V, a, O, s);
    return launch_packed_simt<float, 64>(prm, Q, K, V, a, O, s);
  }
  if (!(prm->flags & TCA_FLAG_PREFILL_SIMT))
    return prm->head_dim == 128 ? launch_packed_tc<128>(prm, Q, K, V, a, O, ws, s) : launch_packed_tc<64>(prm, Q, K, V, a, O, ws, s);
  if (prm->head_dim == 128) return launch_packed_simt<__nv_bfloat16, 128>(prm, Q, K, V, a, O, s);
  return launch_packed_simt<__nv_bfloat16, 64>(prm, Q, K, V, a, O, s);
}
