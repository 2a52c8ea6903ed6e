// tca_attn_paged: attention of one new token per sequence over a paged cache (Eq. 2 with a single query per head),
// grouped query heads, sliding window and sinks, optionally adding each row's attention weight to its mass.
//
// Bound by memory: 2 d elements per visible row, read once for the G heads of the group.  The visible rows of all
// units are cut into one equal share per SM (paged_common.cuh); a CTA streams its share through a shared-memory ring.
//   producer warp   reads the page table four steps ahead and brings one box per page (K or V: all columns of up to
//                   128 rows, 128-byte swizzle; a page without a visible row is not read)
//   8 consumer warps, each 16 rows of every step of 128 and a private online softmax.  bf16: ldmatrix and
//                   mma.sync, the G <= 8 heads are the rows of the A tile (tcgen05 needs 64 of them).  fp32: FP32 pipes,
//                   half a row of K per lane, then D / 32 columns of V per lane.
// At the end of a unit's piece the eight states are merged; a piece that is the whole unit gives the result, others
// partial results that a second kernel merges in order.  Statistics and accumulators are fp32; bf16 weights are rounded
// to bf16 before they meet the values (half a step, 2^-8 of a weight), the row sum adds the unrounded ones.
// A slot nobody sees has no influence whatever it holds: its score is replaced, its value row is not read from the ring.
//
// Weights need the row sums of the whole unit, so the scores are left in the workspace (4 G bytes a row beside 4 d or 8 d)
// and the second kernel turns them into weights.
#include <vector>

#include "bulk_ring.cuh"
#include "paged_common.cuh"
#include "rowslice.cuh"
#include "tensor_map.cuh"

namespace tca {

int check_paged(const tca_params* prm, const tca_paged_desc* c) {
  const int st = check_params(prm);
  if (st != TCA_OK) return st;
  TCA_CHECK_ARG(c && c->k && c->v && c->pos && c->mass && c->table && c->state);
  TCA_CHECK_ARG(aligned(c->k, 16) && aligned(c->v, 16) && aligned(c->state, 16));
  TCA_CHECK_ARG(aligned(c->pos, 4) && aligned(c->mass, 4) && aligned(c->table, 4));
  TCA_CHECK_ARG(c->n_units == int64_t(prm->batch) * prm->n_kv_heads && c->n_pages >= 1 && c->max_pages >= 1);
  if (!is_pow2(c->page_size) || c->page_size < 16 || c->page_size > 256) return TCA_ERR_UNSUPPORTED;
  constexpr int64_t kMost = int64_t(1) << 31;
  if (c->n_pages >= kMost / c->page_size || int64_t(c->max_pages) * c->page_size >= kMost - 256) return TCA_ERR_UNSUPPORTED;
  // steps of all units are counted in 32 bits
  if (c->n_units > 65535 || c->n_units * (int64_t(c->max_pages) * c->page_size / kPagedStep + 3) >= kMost) return TCA_ERR_UNSUPPORTED;
  return TCA_OK;
}

namespace {

constexpr int kConsumers = 256, kThreads = kConsumers + 32, kWarps = kConsumers / 32;
constexpr int kList = 64;
constexpr int kMergeStates = 4;      // warp states in shared memory at a time
constexpr float kLog2e = 1.4426950408889634f;

PagedPlan paged_plan(const tca_params*) {
  PagedPlan p;
  p.n_shares = sm_count();
  p.min_share = 1;
  p.lead = 1;
  return p;
}

PagedWs paged_ws_layout(const tca_params* prm, const tca_paged_desc* c, const PagedPlan& p, bool weights, void* ws) {
  PagedWs w;
  const size_t U = size_t(c->n_units), G = size_t(prm->n_q_heads / prm->n_kv_heads), n = (p.n_shares + U) * G;
  char* base = static_cast<char*>(ws);
  size_t at = kPagedHeaderBytes;
  w.status = reinterpret_cast<int*>(base);
  w.table = reinterpret_cast<int2*>(base + at);
  at += align_up(U * sizeof(int2), 256);
  w.ml = reinterpret_cast<float2*>(base + at);
  at += align_up(n * sizeof(float2), 256);
  w.acc = reinterpret_cast<float*>(base + at);
  at += align_up(n * prm->head_dim * sizeof(float), 256);
  w.score = weights ? reinterpret_cast<float*>(base + at) : nullptr;
  if (weights) at += align_up(size_t(c->n_pages) * c->page_size * G * sizeof(float), 256);
  w.bytes = at;
  return w;
}

template <typename T, int D>
struct PagedRing {
  static constexpr int kBoxes = D * int(sizeof(T)) / 128;        // 128-byte column blocks of a row
  static constexpr int kStageBytes = kPagedStep * 128 * kBoxes;
  static constexpr int kStages = (192 * 1024) / kStageBytes > 12 ? 12 : (192 * 1024) / kStageBytes;
  static constexpr int kScratch = kMergeStates * kMaxGroup * D * 4;
  static constexpr int kSmemBytes = kStages * kStageBytes + kScratch + 1024;
};

// Byte offset of 16-byte piece `piece` of row r of a page box of `rows` rows.
__device__ __forceinline__ uint32_t box_at(int rows, int r, int piece) {
  return uint32_t(piece >> 3) * uint32_t(rows) * 128u + uint32_t(r) * 128u + (uint32_t((piece & 7) ^ (r & 7)) << 4);
}

__device__ __forceinline__ void ldm_x4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldm_x4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A warp's softmax state over its 16 rows of every step.  score(): the rows' scores against the G heads and the new
// maximum and sum; value(): the outputs.  Both get the warp's rows in the ring (base of their page box, its rows, first
// row) and which of the 16 are visible.
template <typename T, int D, int GT>
struct WarpRows;

template <int D, int GT>
struct WarpRows<__nv_bfloat16, D, GT> {
  static constexpr int ND = D / 8, KC = D / 16;
  uint32_t qa[KC][2];
  float o[ND][4], m, l;      // heads gq: entries 0 and 1 (the upper half of the A tile is zero)
  float x[4], corr;          // this step: scores of keys kq, kq + 1, 8 + kq, 9 + kq, in log2 units
  uint32_t pa[2];
  int gq, kq, lane, G;

  __device__ __forceinline__ void begin(const __nv_bfloat16* q, int heads, const float*) {
    lane = threadIdx.x & 31;
    gq = lane >> 2;
    kq = (lane & 3) * 2;
    G = heads;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      qa[c][0] = qa[c][1] = 0u;
      if (gq < G) {
        const __nv_bfloat16* p = q + size_t(gq) * D + c * 16 + kq;
        qa[c][0] = *reinterpret_cast<const uint32_t*>(p);
        qa[c][1] = *reinterpret_cast<const uint32_t*>(p + 8);
      }
    }
#pragma unroll
    for (int j = 0; j < ND; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ void score(uint32_t base, int rows, int r0, unsigned visible, float scale_log2e) {
    float s[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
    const int row = r0 + (lane >> 4) * 8 + (lane & 7), piece = (lane >> 3) & 1;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      uint32_t b[4];
      ldm_x4(b, base + box_at(rows, row, c * 2 + piece));
      const uint32_t a[4] = {qa[c][0], 0u, qa[c][1], 0u};
      mma_16816(s[0], a, b[0], b[1]);
      mma_16816(s[1], a, b[2], b[3]);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = (visible >> ((i >> 1) * 8 + kq + (i & 1))) & 1u ? s[i >> 1][i & 1] * scale_log2e : -INFINITY;
      mx = fmaxf(mx, x[i]);
    }
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
    const float m_new = fmaxf(m, mx), from = m_new == -INFINITY ? 0.f : m_new;
    corr = exp2f(m - from);
    float p[4], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) { p[i] = exp2f(x[i] - from); sum += p[i]; }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    l = l * corr + sum;
    m = m_new;
    pa[0] = ptx::pack_bf16x2(p[0], p[1]);
    pa[1] = ptx::pack_bf16x2(p[2], p[3]);
  }
  // the 16 rows' scores, [head][16]
  __device__ __forceinline__ void leave_scores(float* out) const {
    if (gq >= G) return;
    *reinterpret_cast<float2*>(out + gq * 16 + kq) = make_float2(x[0], x[1]);
    *reinterpret_cast<float2*>(out + gq * 16 + 8 + kq) = make_float2(x[2], x[3]);
  }
  // lanes of a row nobody sees load 16 bytes of zeros instead: zero times an infinity is not zero
  __device__ __forceinline__ void value(uint32_t base, int rows, int r0, unsigned visible, uint32_t zeros) {
    const int r = ((lane >> 3) & 1) * 8 + (lane & 7), half = lane >> 4;
    const uint32_t seen = (visible >> r) & 1u;
    const uint32_t from = seen ? base : zeros;
#pragma unroll
    for (int j = 0; j < ND; j += 2) {
      uint32_t b[4];
      ldm_x4_trans(b, from + seen * box_at(rows, r0 + r, j + half));
      o[j][0] *= corr; o[j][1] *= corr;
      o[j + 1][0] *= corr; o[j + 1][1] *= corr;
      const uint32_t a[4] = {pa[0], 0u, pa[1], 0u};
      mma_16816(o[j], a, b[0], b[1]);
      mma_16816(o[j + 1], a, b[2], b[3]);
    }
  }
  // f(head, column, value): every element of the state that this lane holds
  template <typename F>
  __device__ __forceinline__ void each(F f) {
    if (gq >= G) return;
#pragma unroll
    for (int j = 0; j < ND; ++j) {
      f(gq, j * 8 + kq, o[j][0]);
      f(gq, j * 8 + kq + 1, o[j][1]);
    }
  }
  __device__ __forceinline__ bool stats_lane(int g) const { return g == gq && (lane & 3) == 0; }
  __device__ __forceinline__ float& max_of(int) { return m; }
  __device__ __forceinline__ float& sum_of(int) { return l; }
  // heads whose statistics this lane holds
  __device__ __forceinline__ int head0() const { return gq; }
  __device__ __forceinline__ int head1() const { return min(gq + 1, G); }
};

// fp32: lanes 0-15 hold the first half of the 16 rows' columns for the scores, lanes 16-31 the second; for the outputs a
// lane owns D / 32 columns.  The queries lie in shared memory.  GT: the group, up to a power of two (the heads behind it are zero).
template <int D, int GT>
struct WarpRows<float, D, GT> {
  static constexpr int E = D / 32;
  const float* q;            // shared memory [GT][D]
  float o[GT][E], m[GT], l[GT], x[GT], p[GT], corr[GT];
  int lane, G;

  __device__ __forceinline__ void begin(const float*, int heads, const float* q_shared) {
    lane = threadIdx.x & 31;
    G = heads;
    q = q_shared;
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      m[g] = -INFINITY;
      l[g] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[g][e] = 0.f;
    }
  }
  __device__ __forceinline__ void score(uint32_t base, int rows, int r0, unsigned visible, float scale_log2e) {
    const int r = lane & 15, half = lane >> 4;
    float s[GT];
#pragma unroll
    for (int g = 0; g < GT; ++g) s[g] = 0.f;
#pragma unroll 4
    for (int c = 0; c < D / 8; ++c) {
      const int piece = half * (D / 8) + c;
      float4 k;
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(k.x), "=f"(k.y), "=f"(k.z), "=f"(k.w) : "r"(base + box_at(rows, r0 + r, piece)));
#pragma unroll
      for (int g = 0; g < GT; ++g) {
        const float4 v = *reinterpret_cast<const float4*>(q + g * D + piece * 4);
        s[g] = fmaf(v.w, k.w, fmaf(v.z, k.z, fmaf(v.y, k.y, fmaf(v.x, k.x, s[g]))));
      }
    }
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      s[g] += __shfl_xor_sync(0xffffffffu, s[g], 16);
      x[g] = (visible >> r) & 1u ? s[g] * scale_log2e : -INFINITY;
      float mx = x[g];
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
      const float m_new = fmaxf(m[g], mx), from = m_new == -INFINITY ? 0.f : m_new;
      corr[g] = exp2f(m[g] - from);
      p[g] = exp2f(x[g] - from);
      float sum = p[g];
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      l[g] = l[g] * corr[g] + sum;
      m[g] = m_new;
    }
  }
  __device__ __forceinline__ void leave_scores(float* out) const {
    if (lane >= 16) return;
#pragma unroll
    for (int g = 0; g < GT; ++g)
      if (g < G) out[g * 16 + lane] = x[g];
  }
  __device__ __forceinline__ void value(uint32_t base, int rows, int r0, unsigned visible, uint32_t) {
#pragma unroll
    for (int g = 0; g < GT; ++g)
#pragma unroll
      for (int e = 0; e < E; ++e) o[g][e] *= corr[g];
#pragma unroll 4
    for (int r = 0; r < 16; ++r) {
      if (!((visible >> r) & 1u)) continue;     // the same for the whole warp
      float v[E];
      const uint32_t at = base + box_at(rows, r0 + r, E == 4 ? lane : lane >> 1);
      if constexpr (E == 4)
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(at));
      else
        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(at + (lane & 1) * 8));
#pragma unroll
      for (int g = 0; g < GT; ++g) {
        const float w = __shfl_sync(0xffffffffu, p[g], r);
#pragma unroll
        for (int e = 0; e < E; ++e) o[g][e] = fmaf(w, v[e], o[g][e]);
      }
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int g = 0; g < GT; ++g)
      if (g < G)
#pragma unroll
        for (int e = 0; e < E; ++e) f(g, lane * E + e, o[g][e]);
  }
  __device__ __forceinline__ bool stats_lane(int) const { return lane == 0; }
  __device__ __forceinline__ float& max_of(int g) { return m[g]; }
  __device__ __forceinline__ float& sum_of(int g) { return l[g]; }
  __device__ __forceinline__ int head0() const { return 0; }
  __device__ __forceinline__ int head1() const { return GT; }
};

template <typename T, int D, int GT>
__global__ void __launch_bounds__(kThreads, 1)
paged_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const T* __restrict__ q,
             const __grid_constant__ PagedArgs args, int G, int window, int n_sink, float scale_log2e, PagedPlan plan, PagedWs ws,
             T* __restrict__ O) {
  using Ring = PagedRing<T, D>;
  constexpr int kStages = Ring::kStages;
  extern __shared__ uint8_t paged_smem[];
  uint8_t* ring_buf = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(paged_smem) + 1023) & ~uintptr_t(1023));
  float* scratch = reinterpret_cast<float*>(ring_buf + kStages * Ring::kStageBytes);
  __shared__ BulkRing<kStages> ring;
  __shared__ PagedDeal<kThreads, kList> deal;
  __shared__ int abort_word, stop_word;
  __shared__ __align__(16) uint32_t zeros[4];
  __shared__ __align__(16) float s_q[GT > 0 ? GT * D : 4];
  __shared__ float s_m[kMergeStates][kMaxGroup], s_l[kMergeStates][kMaxGroup];
  __shared__ int group_row[kStages][kWarps];      // a stage's pool rows / 16; -1: not a page of the pool
  volatile int* abort_flag = &abort_word;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    ring.init(kWarps);
    abort_word = 0;
    zeros[0] = zeros[1] = zeros[2] = zeros[3] = 0u;
    ptx::tma_prefetch_desc(&map_k);
    ptx::tma_prefetch_desc(&map_v);
  }
  pdl_wait();
  pdl_launch_dependents();
  if (tid == 0) stop_word = stops_call(*reinterpret_cast<volatile int*>(ws.status));
  const int share = int(blockIdx.x);
  const int box_rows = min(1 << args.page_shift, kPagedStep);      // rows of a box
  int n = 0;                                                       // stages handed over so far
  bool ok = true;
  for (int rank0 = 0;; rank0 += kList) {
    const int n_pieces = deal.deal(args, plan, window, n_sink, share, rank0, ws.table);
    if (stop_word) return;
    const int here = min(kList, n_pieces - rank0);
    if (warp == kWarps) {
      // ------------------------------------------------------------- producer
      // A lane reads the page of one group of 16 rows: of steps 0 .. 3 of a batch, group lane % 8.  The next
      // batch's pages are requested before this one's boxes are issued.
      auto page_of = [&](int i, int s) {          // step s of piece i
        if (i >= here) return -1;
        const PagedPiece& p = deal.list[i];
        if (s + (lane >> 3) >= p.n) return -1;
        const PagedSpan span(p.len, window, n_sink);
        const int slot = span.slot0(p.s0 + s + (lane >> 3)) + (lane & 7) * 16;
        if (!span.any_visible(slot & ~(box_rows - 1), box_rows)) return -1;
        return args.table[size_t(p.u) * args.max_pages + (slot >> args.page_shift)];
      };
      int next_page = page_of(0, 0);
      for (int i = 0; i < here && ok; ++i) {
        const PagedPiece piece = deal.list[i];
        const PagedSpan span(piece.len, window, n_sink);
        for (int s = 0; s < piece.n && ok; s += 4) {
          const int page = next_page;
          next_page = s + 4 < piece.n ? page_of(i, s + 4) : page_of(i + 1, 0);
          for (int b = 0; b < 4 && s + b < piece.n && ok; ++b) {
            const int mine = __shfl_sync(0xffffffffu, page, b * 8 + (lane & 7));
            const int slot = span.slot0(piece.s0 + s + b) + (lane & 7) * 16;
            const bool good = unsigned(mine) < unsigned(args.n_pages);
            const bool wanted = lane < 8 && span.any_visible(slot & ~(box_rows - 1), box_rows);
            if (wanted && !good) report_bounds_ws(ws.status, kBoundsCacheRow, mine);
            const int row = (mine << args.page_shift) + (slot & ((1 << args.page_shift) - 1));
            const bool box = wanted && good && (slot & (box_rows - 1)) == 0;
            const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, box)) * box_rows * 128 * Ring::kBoxes;
            for (int kv = 0; kv < 2 && ok; ++kv, ++n) {
              const int stage = n % kStages;
              if (lane == 0 && n >= kStages) ok = ptx::mbar_wait(&ring.empty[stage], uint32_t(n / kStages - 1) & 1u, abort_flag);
              ok = __shfl_sync(0xffffffffu, ok, 0);
              if (!ok) break;
              if (lane < 8 && kv == 0) group_row[stage][lane] = wanted && good ? row >> 4 : -1;
              __syncwarp();
              if (lane == 0) ptx::mbar_arrive_expect_tx(&ring.full[stage], bytes);
              __syncwarp();
              if (box)
                ptx::tma_load_3d(ring_buf + stage * Ring::kStageBytes + lane * 16 * 128 * Ring::kBoxes, kv ? &map_v : &map_k, 0, row, 0,
                                 &ring.full[stage]);
            }
          }
        }
      }
    } else {
      // ------------------------------------------------------------- consumers
      WarpRows<T, D, GT> rows;
      const int page_in_step = warp * 16 / box_rows, r0 = warp * 16 % box_rows;
      const uint32_t warp_base = ptx::smem_u32(ring_buf) + uint32_t(page_in_step * box_rows * 128 * Ring::kBoxes);
      const uint32_t zero_addr = ptx::smem_u32(zeros);
      for (int i = 0; i < here; ++i) {
        const PagedPiece piece = deal.list[i];
        const PagedSpan span(piece.len, window, n_sink);
        const T* q_unit = q + size_t(piece.u) * G * D;
        if constexpr (GT > 0) {
          for (int j = tid; j < GT * D; j += kConsumers) s_q[j] = j < G * D ? float(q_unit[j]) : 0.f;
          consumer_sync(kConsumers);
        }
        rows.begin(q_unit, G, s_q);
        for (int s = 0; s < piece.n; ++s) {
          const int slot = span.slot0(piece.s0 + s) + warp * 16;
          unsigned visible = span.visible16(slot);
          if (ok) ok = __all_sync(0xffffffffu, ring.wait_full(n, abort_flag));
          const int at = ok ? group_row[n % kStages][warp] : -1;
          if (at < 0) visible = 0;
          if (visible) {
            rows.score(warp_base + (n % kStages) * Ring::kStageBytes, box_rows, r0, visible, scale_log2e);
            if (ws.score) rows.leave_scores(ws.score + size_t(at) * G * 16);
          }
          __syncwarp();
          if (lane == 0) ring.release(n);
          ++n;
          if (ok) ok = __all_sync(0xffffffffu, ring.wait_full(n, abort_flag));
          if (ok && visible) rows.value(warp_base + (n % kStages) * Ring::kStageBytes, box_rows, r0, visible, zero_addr);
          __syncwarp();
          if (lane == 0) ring.release(n);
          ++n;
        }
        // ----------------------------------------------------------- merge the warps' states: 4 .. 7 into 0 .. 3, then those
        const int hs = warp & 3;
        float* mine = scratch + size_t(hs) * G * D;
        if (warp >= 4) {
          rows.each([&](int g, int d, float& v) { mine[g * D + d] = v; });
          for (int g = rows.head0(); g < rows.head1(); ++g)
            if (g < G && rows.stats_lane(g)) { s_m[hs][g] = rows.max_of(g); s_l[hs][g] = rows.sum_of(g); }
        }
        consumer_sync(kConsumers);
        if (warp < 4) {
          float w0[GT > 0 ? GT : 1], w1[GT > 0 ? GT : 1];
#pragma unroll
          for (int k = 0; k < (GT > 0 ? GT : 1); ++k) {
            const int g = rows.head0() + k;
            w0[k] = 1.f;
            w1[k] = 0.f;
            if (g < G) {
              const float ma = rows.max_of(g), mb = s_m[hs][g], M = fmaxf(ma, mb), from = M == -INFINITY ? 0.f : M;
              w0[k] = exp2f(ma - from);
              w1[k] = exp2f(mb - from);
              rows.sum_of(g) = rows.sum_of(g) * w0[k] + s_l[hs][g] * w1[k];
              rows.max_of(g) = M;
            }
          }
          rows.each([&](int g, int d, float& v) {
            const int k = GT > 0 ? g : 0;
            v = v * w0[k] + mine[g * D + d] * w1[k];
            mine[g * D + d] = v;
          });
          __syncwarp();                       // the warp's lanes have read the other state's statistics
          for (int g = rows.head0(); g < rows.head1(); ++g)
            if (g < G && rows.stats_lane(g)) { s_m[hs][g] = rows.max_of(g); s_l[hs][g] = rows.sum_of(g); }
        }
        consumer_sync(kConsumers);
        if (!*abort_flag) {
          const size_t at = size_t(share + piece.u) * G;
          for (int j = tid * 2; j < G * D; j += kConsumers * 2) {
            const int g = j / D, d = j - g * D;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kMergeStates; ++w) M = fmaxf(M, s_m[w][g]);
            const float from = M == -INFINITY ? 0.f : M;
            float a0 = 0.f, a1 = 0.f, l = 0.f;
#pragma unroll
            for (int w = 0; w < kMergeStates; ++w) {
              const float wt = exp2f(s_m[w][g] - from);
              const float2 v = *reinterpret_cast<const float2*>(scratch + (size_t(w) * G + g) * D + d);
              a0 = fmaf(v.x, wt, a0);
              a1 = fmaf(v.y, wt, a1);
              l = fmaf(s_l[w][g], wt, l);
            }
            if (piece.whole) {
              T* out = O + size_t(piece.u) * G * D + j;
              if constexpr (sizeof(T) == 4) *reinterpret_cast<float2*>(out) = make_float2(a0 / l, a1 / l);
              else *reinterpret_cast<uint32_t*>(out) = ptx::pack_bf16x2(a0 / l, a1 / l);
            } else {
              *reinterpret_cast<float2*>(ws.acc + at * D + j) = make_float2(a0, a1);
            }
            if (d == 0) ws.ml[at + g] = make_float2(M, l);
          }
        }
        consumer_sync(kConsumers);            // the states are written over by the next piece
      }
    }
    if (rank0 + kList >= n_pieces) break;
  }
  __syncthreads();
  if (*abort_flag) {
    if (tid == 0) atomicCAS(ws.status, kStatusBounds, kStatusTimeout);
    ptx::abort_teardown(ws.status, tid);
  }
}

// ------------------------------------------------------------------ merge of the partial results; weights
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;

// Blocks below merge_blocks: one warp per (unit, head) merges the unit's partial results in order.  The others (only if
// weights are accumulated): a share of the visible rows each, turning scores into weights.
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads)
paged_join_kernel(const __grid_constant__ PagedArgs args, int G, int window, int n_sink, int merge_blocks, PagedPlan plan, PagedWs ws,
                  float* __restrict__ mass, T* __restrict__ O) {
  __shared__ PagedDeal<kJoinThreads, kList> deal;
  __shared__ float s_lse[kMaxGroup];
  __shared__ int stop_word;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr int E = D / 32;
  if (int(blockIdx.x) < merge_blocks) {
    const int at = int(blockIdx.x) * kJoinWarps + warp, u = at / G, g = at - u * G;
    pdl_wait();
    pdl_launch_dependents();
    if (u >= args.n_units) return;
    const int len = args.state[u].x;
    const int2 where = __ldcg(ws.table + u);
    if (stops_call(__ldcg(ws.status))) return;
    float o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    if (PagedSpan(paged_len(args, len), window, n_sink).n > 0) {
      if (where.y == 0) return;                 // its only share wrote the result
      float m = -INFINITY, l = 0.f;
      for (int c0 = 0; c0 < where.y; c0 += 32) {
        const int cn = min(32, where.y - c0);
        const float2 ml = lane < cn ? __ldcg(ws.ml + size_t(where.x + c0 + lane) * G + g) : make_float2(-INFINITY, 0.f);
        float mn = ml.x;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, off));
        mn = fmaxf(m, mn);
        const float from = mn == -INFINITY ? 0.f : mn, keep = exp2f(m - from), w = exp2f(ml.x - from);
        l *= keep;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= keep;
        const float wl = w * ml.y;
#pragma unroll 8
        for (int c = 0; c < cn; ++c) {
          const float wc = __shfl_sync(0xffffffffu, w, c);
          l += __shfl_sync(0xffffffffu, wl, c);
          const float* a = ws.acc + (size_t(where.x + c0 + c) * G + g) * D + lane * E;
          float v[E];
          if constexpr (E == 4) { const float4 t = __ldcg(reinterpret_cast<const float4*>(a)); v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w; }
          else { const float2 t = __ldcg(reinterpret_cast<const float2*>(a)); v[0] = t.x; v[1] = t.y; }
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] = fmaf(wc, v[e], o[e]);
        }
        m = mn;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] /= l;
    }
    T* out = O + (size_t(u) * G + g) * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      if constexpr (sizeof(T) == 4) *reinterpret_cast<float2*>(out + e) = make_float2(o[e], o[e + 1]);
      else *reinterpret_cast<uint32_t*>(out + e) = ptx::pack_bf16x2(o[e], o[e + 1]);
    }
    return;
  }
  pdl_wait();
  pdl_launch_dependents();
  if (tid == 0) stop_word = stops_call(__ldcg(ws.status));
  const int share = int(blockIdx.x) - merge_blocks;
  const float inv_g = 1.f / float(G);
  for (int rank0 = 0;; rank0 += kList) {
    const int n_pieces = deal.deal(args, plan, window, n_sink, share, rank0, nullptr);
    if (stop_word) return;
    const int here = min(kList, n_pieces - rank0);
    for (int i = 0; i < here; ++i) {
      const PagedPiece p = deal.list[i];
      const PagedSpan span(p.len, window, n_sink);
      __syncthreads();
      if (warp < G) {                           // the row sums of the unit: log2 of the sum over its partial results
        const int2 where = __ldcg(ws.table + p.u);
        float m = -INFINITY, l = 0.f;
        for (int c = lane; c < max(1, where.y); c += 32) {
          const float2 ml = __ldcg(ws.ml + size_t(where.x + c) * G + warp);
          const float mn = fmaxf(m, ml.x), from = mn == -INFINITY ? 0.f : mn;
          l = l * exp2f(m - from) + ml.y * exp2f(ml.x - from);
          m = mn;
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
          const float mo = __shfl_xor_sync(0xffffffffu, m, off), lo = __shfl_xor_sync(0xffffffffu, l, off);
          const float mn = fmaxf(m, mo), from = mn == -INFINITY ? 0.f : mn;
          l = l * exp2f(m - from) + lo * exp2f(mo - from);
          m = mn;
        }
        if (lane == 0) s_lse[warp] = m + log2f(l);
      }
      __syncthreads();
      for (int j = tid; j < p.n * kPagedStep; j += kJoinThreads) {
        const int slot = span.slot0(p.s0 + j / kPagedStep) + j % kPagedStep;
        if (!((span.visible16(slot & ~15) >> (slot & 15)) & 1u)) continue;
        const int row = paged_row(args, p.u, slot);
        if (row < 0) continue;
        const float* x = ws.score + size_t(row >> 4) * G * 16 + (row & 15);
        float sum = 0.f;
        for (int g = 0; g < G; ++g) sum += exp2f(__ldcg(x + g * 16) - s_lse[g]);
        mass[row] += sum * inv_g;
      }
    }
    if (rank0 + kList >= n_pieces) break;
  }
}

// The pool as [column block][row][128 bytes]: boxes of all columns of up to 128 rows.
template <typename T, int D>
bool pool_map(CUtensorMap* out, const void* base, const tca_paged_desc* c) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  constexpr int kCols = 128 / int(sizeof(T));
  cuuint64_t dims[3] = {cuuint64_t(kCols), cuuint64_t(c->n_pages) * c->page_size, cuuint64_t(PagedRing<T, D>::kBoxes)};
  cuuint64_t strides[2] = {cuuint64_t(D) * sizeof(T), 128};
  cuuint32_t box[3] = {cuuint32_t(kCols), cuuint32_t(c->page_size < kPagedStep ? c->page_size : kPagedStep),
                       cuuint32_t(PagedRing<T, D>::kBoxes)};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(out, sizeof(T) == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<void*>(base), dims,
            strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D, int GT>
int launch_paged(const tca_params* prm, const void* q, const tca_paged_desc* c, int n_sink, bool weights, void* O, const PagedPlan& plan,
                 const PagedWs& ws, cudaStream_t s) {
  using Ring = PagedRing<T, D>;
  CUtensorMap mk, mv;
  if (!pool_map<T, D>(&mk, c->k, c) || !pool_map<T, D>(&mv, c->v, c)) return TCA_ERR_CUDA;
  const int G = prm->n_q_heads / prm->n_kv_heads;
  const PagedArgs args = paged_args(c);
  constexpr auto kern = paged_kernel<T, D, GT>;
  if (allow_smem<kern>(Ring::kSmemBytes) != TCA_OK) return TCA_ERR_CUDA;
  const int st = launch_pdl(kern, dim3(unsigned(plan.n_shares)), dim3(kThreads), size_t(Ring::kSmemBytes), s, mk, mv, static_cast<const T*>(q),
                            args, G, prm->window, n_sink, prm->sm_scale * kLog2e, plan, ws, static_cast<T*>(O));
  if (st != TCA_OK) return st;
  const int merge_blocks = int((c->n_units * G + kJoinWarps - 1) / kJoinWarps);
  PagedPlan join = plan;
  join.n_shares = plan.n_shares * 4;
  join.lead = 0;
  return launch_pdl(paged_join_kernel<T, D>, dim3(unsigned(merge_blocks + (weights ? join.n_shares : 0))), dim3(kJoinThreads), size_t(0), s, args,
                    G, prm->window, n_sink, merge_blocks, join, ws, c->mass, static_cast<T*>(O));
}

template <int D>
int launch_paged_f32(const tca_params* prm, const void* q, const tca_paged_desc* c, int n_sink, bool weights, void* O, const PagedPlan& plan,
                     const PagedWs& ws, cudaStream_t s) {
  const int G = prm->n_q_heads / prm->n_kv_heads;
  if (G == 1) return launch_paged<float, D, 1>(prm, q, c, n_sink, weights, O, plan, ws, s);
  if (G == 2) return launch_paged<float, D, 2>(prm, q, c, n_sink, weights, O, plan, ws, s);
  if (G <= 4) return launch_paged<float, D, 4>(prm, q, c, n_sink, weights, O, plan, ws, s);
  return launch_paged<float, D, 8>(prm, q, c, n_sink, weights, O, plan, ws, s);
}

}  // namespace
}  // namespace tca

using namespace tca;

extern "C" size_t tca_attn_paged_workspace_bytes(const tca_params* prm, const tca_paged_desc* c, int32_t accumulate) {
  if (check_paged(prm, c) != TCA_OK) return 0;
  return paged_ws_layout(prm, c, paged_plan(prm), accumulate != 0, nullptr).bytes;
}

extern "C" int tca_attn_paged(const tca_params* prm, const void* q, const tca_paged_desc* c, int32_t n_sink, int32_t accumulate, void* O,
                              void* ws, size_t ws_bytes, void* stream) {
  const int st = check_paged(prm, c);
  if (st != TCA_OK) return st;
  TCA_CHECK_ARG(q && O && ws && n_sink >= 0);
  TCA_CHECK_ARG(aligned(q, 16) && aligned(O, 16) && aligned(ws, 256));
  if (prm->window < 1) return TCA_ERR_UNSUPPORTED;
  const PagedPlan plan = paged_plan(prm);
  const PagedWs lay = paged_ws_layout(prm, c, plan, accumulate != 0, ws);
  if (ws_bytes < lay.bytes) return TCA_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool w = accumulate != 0;
  if (prm->dtype == TCA_F32)
    return prm->head_dim == 128 ? launch_paged_f32<128>(prm, q, c, n_sink, w, O, plan, lay, s) : launch_paged_f32<64>(prm, q, c, n_sink, w, O, plan, lay, s);
  if (prm->head_dim == 128) return launch_paged<__nv_bfloat16, 128, 0>(prm, q, c, n_sink, w, O, plan, lay, s);
  return launch_paged<__nv_bfloat16, 64, 0>(prm, q, c, n_sink, w, O, plan, lay, s);
}

extern "C" int tca_paged_status(const tca_paged_desc* c, void* stream, int64_t* detail) {
  TCA_CHECK_ARG(c && c->state && c->n_units >= 1 && c->n_units < (int64_t(1) << 31));
  std::vector<int32_t> st(size_t(c->n_units) * TCA_PG_STATE_WORDS);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  TCA_CHECK_CUDA(cudaMemcpyAsync(st.data(), c->state, st.size() * sizeof(int32_t), cudaMemcpyDeviceToHost, s));
  TCA_CHECK_CUDA(cudaStreamSynchronize(s));
  for (int64_t u = 0; u < c->n_units; ++u) {
    const int32_t which = st[size_t(u) * TCA_PG_STATE_WORDS + TCA_PG_CHECK];
    if (which != 0) {
      if (detail) { detail[0] = u; detail[1] = which; }
      return TCA_ERR_BOUNDS;
    }
  }
  return TCA_OK;
}
