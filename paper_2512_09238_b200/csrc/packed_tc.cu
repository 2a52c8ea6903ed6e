// tca_attn_packed for bf16: the tensor-core kernel.  One CTA takes 2 P consecutive positions of one
// sequence for all G query heads of one KV head, P = 128 / G: query rows are (position, head) pairs, head
// fastest, so the two blocks of 128 rows are full for any sequence of a few dozen tokens and every K/V
// tile serves 256 rows.  Q comes as one box of P positions x G heads, whatever the strides.
//
// Bound by the chain from a tile's scores to its product (flash_tc.cuh): a prompt of 8192 tokens, 32/8 heads of
// 128, takes 500 us (1100 TFLOP/s, 64 % of the measured burst rate; 477 us at full clock), one of 128K tokens
// 116 ms (1210 TFLOP/s); 24 prompts of 0 to 1024 tokens take 51 us (48 at full clock), where starting and finishing
// an item weighs as much as its tiles.
#include "flash_tc.cuh"
#include "packed_common.cuh"

namespace tca {
namespace {

// Words of the 256-byte workspace: 0 sticky status, then the item counter and the number of CTAs that left,
// both zero between calls.
constexpr int kCounterWord = 16, kLeftWord = 32;

struct PackedItem {
  int64_t row0;
  int len, p0, kvh;
};

template <int D>
struct PackedTcSrc {
  using Item = PackedItem;
  const CUtensorMap *mq, *mk, *mv;
  const __nv_bfloat16* V;
  __nv_bfloat16* O;
  const PackedArgs* a;
  int G, P, max_tiles, unit_major;
  int64_t row0;
  int len, p0, kvh;

  PackedFinder finder;      // the producer warp's
  int* held;

  __device__ __forceinline__ void begin(int lane) { finder.read(*a, 2 * P, lane, held); first = true; }
  // A CTA takes the item of its own number, then whichever is next (a counter in the workspace, asked while
  // the item before is still being worked on): longest first, so that the last ones to finish work on short
  // ones.  (Dealt in turn, the last CTA of a batch of 24 chat prompts finished 19 % after the mean: 50.3 us
  // against 48.1; a prompt of 128K tokens 119 against 115 ms.  What an item computes does not depend on who
  // takes it.)  Two orders, see launch_packed_tc; with the heads one after another the numbers past a head's
  // last item are skipped.
  unsigned* counter;
  bool first;
  __device__ __forceinline__ bool find(int, int lane, Item& it) {
    for (;;) {
      int i = int(blockIdx.x);
      if (!first && max_tiles * a->n_kv_heads <= int(gridDim.x)) return false;   // a CTA for every item
      if (!first) i = int(gridDim.x) + int(__shfl_sync(0xffffffffu, lane == 0 ? atomicAdd(counter, 1u) : 0u, 0));
      first = false;
      if (i >= max_tiles * a->n_kv_heads) return false;
      it.kvh = unit_major ? i / max_tiles : i % a->n_kv_heads;
      int tile;
      if (!finder.find(*a, unit_major ? i % max_tiles : i / a->n_kv_heads, 2 * P, lane, it.row0, it.len, tile)) {
        if (unit_major) continue;
        return false;                        // the numbers without an item are the last ones
      }
      it.p0 = tile * 2 * P;
      return true;
    }
  }
  __device__ __forceinline__ void set(const Item& it) { row0 = it.row0; len = it.len; p0 = it.p0; kvh = it.kvh; }

  __device__ __forceinline__ int last_pos(int h) const { return min(p0 + (h + 1) * P, len) - 1; }
  __device__ __forceinline__ int tiles(int h) const { return p0 + h * P < len ? last_pos(h) / kTcKeys + 1 : 0; }
  __device__ __forceinline__ int q_bytes(int) const { return D * 2 * G * P; }
  __device__ __forceinline__ void load_q(int h, uint8_t* dst, uint64_t* bar) const {
    for (int half = 0; half < D / 64; ++half)
      ptx::tma_load_3d(dst + half * kTcHalfBytes, mq, half * 64, kvh * G, int(row0) + p0 + h * P, bar);
  }
  __device__ __forceinline__ void load(int t, bool is_v, uint8_t* dst, uint64_t* bar) const {
    for (int half = 0; half < D / 64; ++half)
      ptx::tma_load_3d(dst + half * kTcHalfBytes, is_v ? mv : mk, half * 64, int(row0) + t * kTcKeys, kvh, bar);
  }
  int dp, g;                // this thread's row: position and head within the block
  __device__ __forceinline__ void begin_row(int row) { dp = row / G; g = row % G; }
  __device__ __forceinline__ int row_key(int h) const { return min(p0 + h * P + dp, last_pos(h)); }
  __device__ __forceinline__ int last(int key, int t) const { return key - t * kTcKeys; }
  __device__ __forceinline__ int whole_tiles() const { return p0 / kTcKeys; }
  __device__ __forceinline__ int keys(int h, int t) const { return min(kTcKeys, last_pos(h) + 1 - t * kTcKeys); }
  // From the tile that holds p0 on, some row does not see some key (at most two tiles: 2 P <= 128, or
  // P = 128 with p0 a multiple of 256).  Rows past the last position are nobody's: another sequence's, or
  // none; rows up to p0 are everybody's.
  __device__ __forceinline__ int clean(int t) const {
    return t < p0 / kTcKeys ? -1 : min(kTcKeys, min(p0 + 2 * P, len) - t * kTcKeys);
  }
  __device__ __forceinline__ int scan_from(int t) const { return max(0, p0 + 1 - t * kTcKeys); }
  __device__ __forceinline__ int note_slot(int t) const { return t - p0 / kTcKeys; }

  template <typename Read>
  __device__ __forceinline__ void store(int h, bool seen, float, float l, const uint32_t* dirty, Read read) const {
    if (!seen) return;
    const int pos = p0 + h * P + dp;
    const bool mine = dp < P && pos < len;
    const float inv = 1.f / l;
    __nv_bfloat16* out = O + (kvh * G + g) * a->o.head + (row0 + pos) * a->o.row;
    const TcRowOut rows_out(mine ? out : nullptr);
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t v[32];
      read(c, v);
      ptx::tc_wait_ld();
#pragma unroll
      for (int k = 0; k < 16; ++k)
        v[k] = ptx::pack_bf16x2(__uint_as_float(v[2 * k]) * inv, __uint_as_float(v[2 * k + 1]) * inv);
      rows_out.store16(v, c * 64);
    }
    if (dirty) {   // non-finite values of masked tiles, kept out of the product, are added to the rows that see them
      __syncwarp();                       // a row has been written by the four lanes of its quad
      if (!mine) return;
#pragma unroll 1
      for (int i = 0; i < 8; ++i)
        for (uint32_t bits = dirty[i]; bits; bits &= bits - 1) {
          const int key = (p0 / kTcKeys + (i >> 2)) * kTcKeys + (i & 3) * 32 + __ffs(bits) - 1;
          if (key > pos) break;
          const __nv_bfloat16* src = V + kvh * a->v.head + (row0 + key) * a->v.row;
#pragma unroll 1
          for (int k = 0; k < D; ++k) {
            const float x = __bfloat162float(src[k]);
            if (!isfinite(x)) out[k] = __float2bfloat16_rn(__bfloat162float(out[k]) + x);
          }
        }
    }
  }
};

template <int D>
__global__ void __launch_bounds__(kTcThreads, 1)
packed_tc_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                 const __grid_constant__ CUtensorMap mv, const __nv_bfloat16* __restrict__ V,
                 const __grid_constant__ PackedArgs args, int max_tiles, int unit_major, float scale_log2e,
                 __nv_bfloat16* __restrict__ O, int* __restrict__ status) {
  extern __shared__ uint8_t packed_tc_smem[];
  __shared__ TcShared<PackedItem> sh;
  __shared__ int held[PackedFinder::kHeld];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(packed_tc_smem) + 1023) & ~uintptr_t(1023));
  if (threadIdx.x == 0) {
    ptx::tma_prefetch_desc(&mq);
    ptx::tma_prefetch_desc(&mk);
    ptx::tma_prefetch_desc(&mv);
  }
  flash_tc_setup<D>(smem, &sh);
  pdl_wait();
  pdl_launch_dependents();
  PackedTcSrc<D> src;
  src.mq = &mq; src.mk = &mk; src.mv = &mv;
  src.V = V; src.O = O; src.a = &args;
  src.G = args.n_q_heads / args.n_kv_heads;
  src.P = kTcRows / src.G;
  src.held = held;
  src.max_tiles = max_tiles;
  src.unit_major = unit_major;
  src.counter = reinterpret_cast<unsigned*>(status) + kCounterWord;
  flash_tc<D, true>(src, smem, &sh, scale_log2e, status);
  if (threadIdx.x == 0 && max_tiles * args.n_kv_heads > int(gridDim.x)) {   // the last CTA to leave puts the counter back for the next call
    unsigned* left = reinterpret_cast<unsigned*>(status) + kLeftWord;
    __threadfence();
    if (atomicAdd(left, 1u) == gridDim.x - 1) {
      *src.counter = 0;
      *left = 0;
    }
  }
}

}  // namespace

template <int D>
int launch_packed_tc(const tca_params* prm, const void* Q, const void* K, const void* V, const PackedArgs& a, void* O,
                     void* ws, cudaStream_t s) {
  const int G = a.n_q_heads / a.n_kv_heads, P = kTcRows / G;
  const int64_t max_tiles = packed_max_tiles(a.rows, a.n_seq, 2 * P);
  if (max_tiles * a.n_kv_heads >= (int64_t(1) << 31) - 65536)   // item numbers, one round past the end, are 32-bit
    return TCA_ERR_UNSUPPORTED;
  CUtensorMap mq, mk, mv;
  if (!encode_map_3d(&mq, Q, D, a.n_q_heads, a.rows, a.q.head, a.q.row, G, P) ||
      !encode_map_3d(&mk, K, D, a.rows, a.n_kv_heads, a.k.row, a.k.head, kTcKeys, 1) ||
      !encode_map_3d(&mv, V, D, a.rows, a.n_kv_heads, a.v.row, a.v.head, kTcKeys, 1))
    return TCA_ERR_CUDA;
  auto kern = packed_tc_kernel<D>;
  if (allow_smem<packed_tc_kernel<D>>(TcLayout<D>::bytes) != TCA_OK) return TCA_ERR_CUDA;
  // Items of all heads in one order balance best, but then the resident CTAs read all heads' keys at once;
  // when those are more than half of the L2 the heads go one after another (128K tokens, 8 heads: 120
  // against 135 ms).  Not with more sequences than the finder sorts: their keys are read once or
  // twice anyway if they are short (500 prompts of up to 200 tokens: 460 against 590 us).  A long prompt among so
  // many pays for it: 128K tokens among 127 prompts of 20 tokens 116 ms, among 128 or more 119 to 121 ms.
  const int unit_major = a.n_seq <= PackedFinder::kHeld && a.rows * a.n_kv_heads * D * 4 > l2_bytes() / 2 ? 1 : 0;
  const int64_t items = max_tiles * a.n_kv_heads, sms = sm_count();
  return launch_pdl(kern, dim3(unsigned(items < sms ? items : sms)), dim3(kTcThreads), size_t(TcLayout<D>::bytes), s, mq, mk,
                    mv, static_cast<const __nv_bfloat16*>(V), a, int(max_tiles), unit_major,
                    prm->sm_scale * 1.4426950408889634f, static_cast<__nv_bfloat16*>(O), static_cast<int*>(ws));
}

template int launch_packed_tc<64>(const tca_params*, const void*, const void*, const void*, const PackedArgs&, void*, void*,
                                  cudaStream_t);
template int launch_packed_tc<128>(const tca_params*, const void*, const void*, const void*, const PackedArgs&, void*, void*,
                                   cudaStream_t);

}  // namespace tca
