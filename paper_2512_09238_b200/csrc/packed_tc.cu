// tca_attn_packed and tca_attn_window for bf16: the tensor-core kernel.  One CTA takes 2 P consecutive positions of one
// sequence for all G query heads of one KV head, P = 128 / G: query rows are (position, head) pairs, head
// fastest, so the two blocks of 128 rows are full for any sequence of a few dozen tokens and every K/V
// tile serves 256 rows.  Q comes as one box of P positions x G heads, whatever the strides.
//
// Bound by the chain from a tile's scores to its product (flash_tc.cuh): a prompt of 8192 tokens, 32/8 heads of
// 128, takes 500 us (1100 TFLOP/s, 64 % of the measured burst rate; 477 us at full clock), one of 128K tokens
// 116 ms (1210 TFLOP/s); 24 prompts of 0 to 1024 tokens take 51 us (48 at full clock), where starting and finishing
// an item weighs as much as its tiles.
//
// With a window the tiles are fewer and of two kinds (WindowTiles): 24 prompts of 0 to 2048 tokens under 512 keys and 16 sinks take
// 96 us (items of 5 tiles: 17000 clocks, and 5000 for the end of one); 32768 tokens and two shorter prompts under 4096 keys
// 1.80 to 1.90 ms (1.09 to 1.15 PFLOP/s).
#include "flash_tc.cuh"
#include "packed_common.cuh"

namespace tca {
namespace {

// Words of the 256-byte workspace: 0 sticky status, then the item counter and the number of CTAs that left,
// both zero between calls.
constexpr int kCounterWord = 16, kLeftWord = 32;

constexpr int kHalf = kTcKeys / 2;

// A run of half tiles that lie one behind the other: half i >= first begins at key 64 i + shift.
struct KeyRun {
  int first, shift;
};

// The keys of query positions p0 .. last of a sequence under a window of w keys and S sinks, in halves of tiles (64
// keys), in the order in which they are taken: those that every row sees whole come first (flash_tc.cuh).  The band
// begins at key b0: the first that the first row's window holds, or 0 where the sinks reach it; sinks in front of the
// band have halves of their own.  Halves, because the band's two edges, 2 P keys each, and the sinks then share tiles: 512
// keys and 16 sinks for 64 positions are 5 tiles instead of 6.
struct WindowTiles {
  int n, whole;            // halves; of them whole
  KeyRun run[5];           // whole sink halves, whole band halves, the rest of the sinks, lower and upper edge of the band
  int rest;                // keys of the third run's half
  __host__ __device__ WindowTiles() {}
  __host__ __device__ WindowTiles(int p0, int last, int w, int sinks) {
    const int c_lo = p0 - w + 1 > 0 ? p0 - w + 1 : 0;     // first key of the first row's window
    const int all_lo = last - w + 1 > 0 ? last - w + 1 : 0;   // first key of every row's window
    const bool apart = sinks < c_lo;
    const int b0 = apart ? c_lo : 0;
    const int n_band = (last - b0) / kHalf + 1;
    const int to_diag = (p0 + 1 - b0) / kHalf;             // band halves in front of the diagonal
    const int in_sinks = apart ? 0 : sinks / kHalf < to_diag ? sinks / kHalf : to_diag;
    const int from = (all_lo - b0 + kHalf - 1) / kHalf;
    const int a = from > in_sinks ? from : in_sinks;       // band halves [a, to_diag) are whole
    const int w0 = apart ? sinks / kHalf : in_sinks, w1 = to_diag > a ? to_diag - a : 0;
    rest = apart ? sinks % kHalf : 0;
    const int r = rest > 0 ? 1 : 0;
    const int low = (a < n_band ? a : n_band) - in_sinks;  // halves [in_sinks, a): some row's window begins inside
    const int up = to_diag > in_sinks + low ? to_diag : in_sinks + low;
    whole = w0 + w1;
    n = whole + r + low + (n_band - up);
    run[0] = KeyRun{0, 0};
    run[1] = KeyRun{w0, b0 + (a - w0) * kHalf};
    run[2] = KeyRun{whole, (w0 - whole) * kHalf};
    run[3] = KeyRun{whole + r, b0 + (in_sinks - whole - r) * kHalf};
    run[4] = KeyRun{whole + r + low, b0 + (up - whole - r - low) * kHalf};
  }
  __host__ __device__ int key0(int half) const {           // of a half that is not there: the last one's
    const int i = half < n ? half : n - 1;
    int shift = 0;
    for (int k = 1; k < 5; ++k) shift = i >= run[k].first ? run[k].shift : shift;
    return i * kHalf + shift;
  }
  __host__ __device__ bool is_rest(int half) const { return rest > 0 && half == whole; }
  // rows of a half that somebody sees, and from which on some row may not see one
  __host__ __device__ int seen(int half, int last) const {
    if (half >= n) return 0;
    if (is_rest(half)) return rest;
    const int k = last + 1 - key0(half);
    return k < kHalf ? k : kHalf;
  }
  __host__ __device__ int scan_from(int half, int p0, int last, int w) const {
    if (half < whole || half >= n || is_rest(half)) return kHalf;
    const int k0 = key0(half);
    if (half < run[4].first || k0 <= last - w) return 0;
    return p0 + 1 > k0 ? p0 + 1 - k0 : 0;
  }
  // Which of keys 32 c .. 32 c + 31 of tile t the row at `pos` sees.
  __host__ __device__ static uint32_t below(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }
  __host__ __device__ uint32_t seen_bits(int pos, int t, int c, int w, int sinks) const {
    const int half = 2 * t + (c >> 1), off = (c & 1) * 32;
    if (half >= n) return 0u;
    if (is_rest(half)) return below(rest - off);
    const int k0 = key0(half) + off;
    return below(pos + 1 - k0) & ~(below(pos - w + 1 - k0) & ~below(sinks - k0));
  }
};

template <bool kWindow>
struct PackedItem {
  int64_t row0;
  int len, p0, kvh;
};
template <>
struct PackedItem<true> {
  int64_t row0;
  int len, p0, kvh;
  WindowTiles tiles;
};

template <int D, bool kWindow>
struct PackedTcSrc {
  using Item = PackedItem<kWindow>;
  static constexpr int kNoted = kWindow ? 6 : 2;
  static constexpr bool kBits = kWindow;
  const CUtensorMap *mq, *mk, *mv;
  const __nv_bfloat16* V;
  __nv_bfloat16* O;
  const PackedArgs* a;
  int G, P, max_tiles, unit_major;
  int64_t row0;
  int len, p0, kvh;
  WindowTiles win;          // kWindow only

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
      if constexpr (kWindow) it.tiles = WindowTiles(it.p0, min(it.p0 + 2 * P, it.len) - 1, a->window, a->n_sink);
      return true;
    }
  }
  __device__ __forceinline__ void set(const Item& it) {
    row0 = it.row0; len = it.len; p0 = it.p0; kvh = it.kvh;
    if constexpr (kWindow) win = it.tiles;
  }

  __device__ __forceinline__ int last_pos(int h) const { return min(p0 + (h + 1) * P, len) - 1; }
  __device__ __forceinline__ int tiles(int h) const {
    if (p0 + h * P >= len) return 0;
    if constexpr (kWindow) return (win.n + 1) / 2;
    return last_pos(h) / kTcKeys + 1;
  }
  __device__ __forceinline__ int q_bytes(int) const { return D * 2 * G * P; }
  __device__ __forceinline__ void load_q(int h, uint8_t* dst, uint64_t* bar) const {
    for (int half = 0; half < D / 64; ++half)
      ptx::tma_load_3d(dst + half * kTcHalfBytes, mq, half * 64, kvh * G, int(row0) + p0 + h * P, bar);
  }
  __device__ __forceinline__ void load(int t, bool is_v, uint8_t* dst, uint64_t* bar) const {
    for (int part = 0; part < (kWindow ? 2 : 1); ++part) {   // boxes of 64 rows or of 128
      const int row = int(row0) + (kWindow ? win.key0(2 * t + part) : t * kTcKeys);
      for (int half = 0; half < D / 64; ++half)
        ptx::tma_load_3d(dst + half * kTcHalfBytes + part * (kTcHalfBytes / 2), is_v ? mv : mk, half * 64, row, kvh, bar);
    }
  }
  int dp, g;                // this thread's row: position and head within the block
  __device__ __forceinline__ void begin_row(int row) { dp = row / G; g = row % G; }
  __device__ __forceinline__ int row_key(int h) const { return min(p0 + h * P + dp, last_pos(h)); }
  __device__ __forceinline__ int last(int key, int t) const { return key - t * kTcKeys; }
  __device__ __forceinline__ uint32_t seen_bits(int key, int t, int c) const { return win.seen_bits(key, t, c, a->window, a->n_sink); }
  __device__ __forceinline__ int whole_tiles() const {
    if constexpr (kWindow) return win.whole / 2;
    return p0 / kTcKeys;
  }
  __device__ __forceinline__ int keys(int h, int t) const {
    if constexpr (kWindow) return kTcKeys;
    return min(kTcKeys, last_pos(h) + 1 - t * kTcKeys);
  }
  // From the tile that holds p0 on, some row does not see some key (at most two tiles: 2 P <= 128, or
  // P = 128 with p0 a multiple of 256; with a window at most six).  Rows past the last position are nobody's: another
  // sequence's, or none; rows up to p0 are everybody's.
  __device__ __forceinline__ int clean(int t) const {      // window: of half t
    if constexpr (kWindow) return t / 2 < whole_tiles() ? -1 : win.seen(t, last_pos(1));
    return t < whole_tiles() ? -1 : min(kTcKeys, min(p0 + 2 * P, len) - t * kTcKeys);
  }
  __device__ __forceinline__ int scan_from(int t) const {
    if constexpr (kWindow) return win.scan_from(t, p0, last_pos(1), a->window);
    return max(0, p0 + 1 - t * kTcKeys);
  }
  __device__ __forceinline__ int note_slot(int t) const { return t - whole_tiles(); }

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
      for (int i = 0; i < 4 * kNoted; ++i)
        for (uint32_t bits = dirty[i]; bits; bits &= bits - 1) {
          const int bit = __ffs(bits) - 1, t = whole_tiles() + (i >> 2);
          int key = t * kTcKeys + (i & 3) * 32 + bit;
          if constexpr (kWindow) {
            if (!((seen_bits(pos, t, i & 3) >> bit) & 1u)) continue;
            key = win.key0(2 * t + ((i >> 1) & 1)) + (i & 1) * 32 + bit;
          } else if (key > pos) {
            break;
          }
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

template <int D, bool kWindow>
__global__ void __launch_bounds__(kTcThreads, 1)
packed_tc_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                 const __grid_constant__ CUtensorMap mv, const __nv_bfloat16* __restrict__ V,
                 const __grid_constant__ PackedArgs args, int max_tiles, int unit_major, float scale_log2e,
                 __nv_bfloat16* __restrict__ O, int* __restrict__ status) {
  extern __shared__ uint8_t packed_tc_smem[];
  __shared__ TcShared<PackedItem<kWindow>, PackedTcSrc<D, kWindow>::kNoted> sh;
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
  PackedTcSrc<D, kWindow> src;
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

template <int D, bool kWindow>
int launch_packed_tc(const tca_params* prm, const void* Q, const void* K, const void* V, const PackedArgs& a, void* O,
                     void* ws, cudaStream_t s) {
  const int G = a.n_q_heads / a.n_kv_heads, P = kTcRows / G;
  const int64_t max_tiles = packed_max_tiles(a.rows, a.n_seq, 2 * P);
  if (max_tiles * a.n_kv_heads >= (int64_t(1) << 31) - 65536)   // item numbers, one round past the end, are 32-bit
    return TCA_ERR_UNSUPPORTED;
  CUtensorMap mq, mk, mv;
  if (!encode_map_3d(&mq, Q, D, a.n_q_heads, a.rows, a.q.head, a.q.row, G, P) ||
      !encode_map_3d(&mk, K, D, a.rows, a.n_kv_heads, a.k.row, a.k.head, kWindow ? kHalf : kTcKeys, 1) ||
      !encode_map_3d(&mv, V, D, a.rows, a.n_kv_heads, a.v.row, a.v.head, kWindow ? kHalf : kTcKeys, 1))
    return TCA_ERR_CUDA;
  auto kern = packed_tc_kernel<D, kWindow>;
  if (allow_smem<packed_tc_kernel<D, kWindow>>(TcLayout<D>::bytes) != TCA_OK) return TCA_ERR_CUDA;
  // Items of all heads in one order balance best, but then the resident CTAs read all heads' keys at once;
  // when those are more than half of the L2 the heads go one after another (128K tokens, 8 heads: 120
  // against 135 ms).  Not with more sequences than the finder sorts: their keys are read once or
  // twice anyway if they are short (500 prompts of up to 200 tokens: 460 against 590 us).  A long prompt among so
  // many pays for it: 128K tokens among 127 prompts of 20 tokens 116 ms, among 128 or more 119 to 121 ms.
  // Under a window neighbouring items share their keys, so all heads at once need little of the L2.
  const int unit_major = !kWindow && a.n_seq <= PackedFinder::kHeld && a.rows * a.n_kv_heads * D * 4 > l2_bytes() / 2 ? 1 : 0;
  const int64_t items = max_tiles * a.n_kv_heads, sms = sm_count();
  return launch_pdl(kern, dim3(unsigned(items < sms ? items : sms)), dim3(kTcThreads), size_t(TcLayout<D>::bytes), s, mq, mk,
                    mv, static_cast<const __nv_bfloat16*>(V), a, int(max_tiles), unit_major,
                    prm->sm_scale * 1.4426950408889634f, static_cast<__nv_bfloat16*>(O), static_cast<int*>(ws));
}

#define TCA_INSTANTIATE(D, W)                                                                                                   \
  template int launch_packed_tc<D, W>(const tca_params*, const void*, const void*, const void*, const PackedArgs&, void*, void*, \
                                      cudaStream_t);
TCA_INSTANTIATE(64, false)
TCA_INSTANTIATE(128, false)
TCA_INSTANTIATE(64, true)
TCA_INSTANTIATE(128, true)
#undef TCA_INSTANTIATE

}  // namespace tca
