// tca_attn_paged: attention of one new token per sequence over a paged cache (Eq. 2 with a single query per head),
// grouped query heads, sliding window and sinks, optionally adding each row's attention weight to its mass.
//
// Bound by memory: 2 d elements per visible row, read once for the G heads of the group.  The visible rows of all
// units are cut into one equal share per SM (paged_common.cuh); a CTA streams its share through a shared-memory ring.
//   producer warp   reads the page table three batches of four steps ahead and brings one box per page (K or V: all
//                   columns of up to 128 rows, 128-byte swizzle; a page without a visible row is not read)
//   two teams of 4 consumer warps, which take the pieces of the share in turn; a warp has 32 rows of every step of 128
//                   and a private online softmax.  bf16: ldmatrix and mma.sync, the G <= 8 heads are the columns of the
//                   products (tcgen05 needs 64 rows of queries).  fp32: FP32 pipes, a row of K per lane, then D / 32
//                   columns of V per lane.
// At the end of a unit's piece the four states are merged; a piece that is the whole unit gives the result, others
// partial results, which whoever brings the unit's last one merges in order.  Statistics and accumulators are fp32; bf16
// weights are rounded to bf16 before they meet the values (half a step, 2^-8 of a weight), the row sum adds the
// unrounded ones.  A slot nobody sees has no influence whatever it holds: its score is replaced, its value row is not
// read from the ring.
//
// Weights need the row sums of the whole unit, so the scores are left in the workspace (4 G bytes a row beside 4 d or 8 d)
// and a second kernel turns them into weights; it merges the partial results as well, which costs nothing there (in the
// first kernel, 2.5 us).
//
// Measured, 32/8 heads of 128, bf16, a captured call: one sequence of 700 rows 8.3 us (latency: about 5 us until the first rows
// are there); 4 sequences of up to 64K rows (249 MB) 41 us over the same cache again, 47 over caches that change
// (5.3 TB/s); 256 sequences of 500 to 1000 rows (790 MB) 127 us (6.2 TB/s), with weights 155; 64 sequences of up to 4K
// rows (138 MB) with weights 36, of which the second kernel is 8.
#include "bulk_ring.cuh"
#include "paged_common.cuh"
#include "rowslice.cuh"
#include "team.cuh"
#include "tensor_map.cuh"

namespace tca {

int check_paged(const tca_params* prm, const tca_paged_desc* c) {
  const int st = check_params(prm);
  if (st != TCA_OK) return st;
  TCA_CHECK_ARG(c && c->k && c->v && c->pos && c->mass && c->table && c->state);
  TCA_CHECK_ARG(aligned(c->k, 16) && aligned(c->v, 16) && aligned(c->state, 16) && aligned(c->pos, 16) && aligned(c->mass, 16));
  TCA_CHECK_ARG(aligned(c->table, 4));
  TCA_CHECK_ARG(c->n_units == int64_t(prm->batch) * prm->n_kv_heads && c->n_pages >= 1 && c->max_pages >= 1);
  if (!is_pow2(c->page_size) || c->page_size < 16 || c->page_size > 256) return TCA_ERR_UNSUPPORTED;
  constexpr int64_t kMost = int64_t(1) << 31;
  if (c->n_pages >= kMost / c->page_size || int64_t(c->max_pages) * c->page_size >= kMost - 256) return TCA_ERR_UNSUPPORTED;
  // steps of all units are counted in 32 bits
  if (c->n_units > 65535 || c->n_units * (int64_t(c->max_pages) * c->page_size / kPagedStep + 3) >= kMost) return TCA_ERR_UNSUPPORTED;
  return TCA_OK;
}

namespace {

constexpr int kConsumers = 128, kWarps = kConsumers / 32;   // of a team
constexpr int kWarpRows = kPagedStep / kWarps;      // of a step
static_assert(kWarpRows == 32, "two groups of 16 rows, one lane per row");
constexpr int kList = 128;           // pieces of a round
constexpr int kPageBatches = 3;      // batches of page numbers on their way
constexpr int kGroups = kPagedStep / 16;            // groups of 16 rows of a step: none is on two pages
__host__ __device__ constexpr int state_row(int d) { return d + 4; }   // floats per head of a warp's state in shared memory
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kL2Share = 0.45;

PagedWs paged_ws_layout(const tca_params* prm, const tca_paged_desc* c, bool weights, void* ws) {
  PagedWs w;
  const size_t U = size_t(c->n_units), G = size_t(prm->n_q_heads / prm->n_kv_heads), n = (size_t(sm_count()) + U) * G;
  char* base = static_cast<char*>(ws);
  size_t at = kPagedHeaderBytes;
  w.status = reinterpret_cast<int*>(base);
  w.tickets = reinterpret_cast<int*>(base + at);
  at += align_up(size_t(sm_count()) * sizeof(int), 256);
  w.records = reinterpret_cast<PagedRecord*>(base + at);
  at += align_up(size_t(sm_count()) * sizeof(PagedRecord), 256);
  w.ml = reinterpret_cast<float2*>(base + at);
  at += align_up(n * sizeof(float2), 256);
  w.acc = reinterpret_cast<float*>(base + at);
  at += align_up(n * prm->head_dim * sizeof(float), 256);
  w.score = nullptr;
  w.steps = nullptr;
  if (weights) {
    w.score = reinterpret_cast<float*>(base + at);
    at += align_up(size_t(c->n_pages) * c->page_size * G * sizeof(float), 256);
    w.steps = reinterpret_cast<PagedStepRecord*>(base + at);
    at += align_up(U * (size_t(c->max_pages) * c->page_size / kPagedStep + 2) * sizeof(PagedStepRecord), 256);
  }
  w.bytes = at;
  return w;
}

// GT: heads of the group, at most.
template <typename T, int D, int GT>
struct PagedRing {
  static constexpr int kBoxes = D * int(sizeof(T)) / 128;        // 128-byte column blocks of a row
  static constexpr int kStageBytes = kPagedStep * 128 * kBoxes;
  // Teams of consumers.  They take pieces in turn, so that one streams while the other begins and ends one (3500 clocks for
  // a piece of one step, whose 64 KB take 2300).
  static constexpr int kTeams = kStageBytes == 65536 && GT == 8 ? 1 : 2;
  static constexpr int kThreads = kTeams * kConsumers + 32;
  static constexpr int kState = kWarps * GT * state_row(D) * 4;  // a team's states
  static constexpr int kQueryBytes = GT * D * int(sizeof(T));
  // Queries of the pieces that the producer is ahead by: a piece has two stages or more.
  static constexpr int queries(int stages) { return stages / 2 + 2; }
  static constexpr int bytes(int stages) { return stages * kStageBytes + kTeams * kState + queries(stages) * kQueryBytes + 1024; }
  static constexpr int most() {
    int n = 2;
    while (n < 12 && bytes(n + 1) <= 227 * 1024 - 5632) ++n;
    return n;
  }
  static constexpr int kStages = most(), kQueries = queries(kStages), kSmemBytes = bytes(kStages);
};

// Barrier of a team.
__device__ __forceinline__ void team_sync(int team) {
  asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(kConsumers) : "memory");
}
__device__ __forceinline__ void cp_async_4(int* smem_dst, const int* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(ptx::smem_u32(smem_dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void cp_async_pending() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }

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
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A warp's softmax state over its 32 rows of every step.  score(): the rows' scores against the G heads and their weights;
// value(): the outputs.  Both get where the warp's two groups of 16 rows lie in the ring (base of their page box, first row
// in it) and which rows are visible.  The maximum that weights refer to moves only when a score is more than 2^8 above it,
// so that a step needs one vote and no reduction; sums stay per lane until the piece is done.
struct WarpPlace {
  uint32_t base[2];
  int r0[2], box_rows;
};
constexpr float kGrow = 8.f;

template <typename T, int D, int GT>
struct WarpRows;

// bf16: S^T = K Q^T and O^T = V^T P^T, so that the A tiles are full (16 keys, 16 columns) and the 8 columns of B are the
// heads; P^T is S^T transposed within 8 x 8 blocks.  A lane holds keys lane / 4 (+ 8) of heads 2 (lane % 4) (+ 1) of the
// scores, columns 16 j + lane / 4 (+ 8) of the same heads of the outputs.
template <int D, int GT>
struct WarpRows<__nv_bfloat16, D, GT> {
  static constexpr int KC = D / 16;
  uint32_t q[KC][2];
  float o[KC][4], m[2], l[2];
  float x[2][4];             // [group of rows][key, head]: in log2 units
  uint32_t p[2][2];
  int lane, G;

  __device__ __forceinline__ void begin(const __nv_bfloat16* queries, int heads) {   // shared memory [heads][D]
    lane = threadIdx.x & 31;
    G = heads;
    const int g = lane >> 2, k = (lane & 3) * 2;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const __nv_bfloat16* at = queries + min(g, G - 1) * D + c * 16 + k;
      q[c][0] = *reinterpret_cast<const uint32_t*>(at);
      q[c][1] = *reinterpret_cast<const uint32_t*>(at + 8);
      o[c][0] = o[c][1] = o[c][2] = o[c][3] = 0.f;
    }
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }
  __device__ __forceinline__ void score(const WarpPlace& w, uint32_t stage, unsigned visible, float scale_log2e) {
    float s[2][2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][0][i] = s[t][1][i] = 0.f;
    // A = 16 keys x 16 columns: matrices (keys 0-7, columns 0-7), (8-15, 0-7), (0-7, 8-15), (8-15, 8-15)
    // (all loads first: a load waits its turn behind the product before it.  A group nobody sees is read for nothing)
    const int r = lane & 15, piece = lane >> 4;
    uint32_t a[2][KC][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < KC; ++c) ldm_x4(a[t][c], w.base[t] + stage + box_at(w.box_rows, w.r0[t] + r, c * 2 + piece));
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t) mma_16816(s[t][c & 1], a[t][c], q[c][0], q[c][1]);
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = 16 * t + (lane >> 2) + (i >> 1) * 8;
        x[t][i] = (visible >> key) & 1u ? (s[t][0][i] + s[t][1][i]) * scale_log2e : -INFINITY;
        top[i & 1] = fmaxf(top[i & 1], x[t][i]);
      }
    if (__any_sync(0xffffffffu, top[0] > m[0] + kGrow || top[1] > m[1] + kGrow)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], off));
        if (top[h] > m[h] + kGrow) {
          const float alpha = ptx::fast_exp2(m[h] - top[h]);
          l[h] *= alpha;
#pragma unroll
          for (int c = 0; c < KC; ++c) { o[c][h] *= alpha; o[c][2 + h] *= alpha; }
          m[h] = top[h];
        }
      }
    }
    const float from[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        e[i] = ptx::fast_exp2(x[t][i] - from[i & 1]);
        l[i & 1] += e[i];
      }
#pragma unroll
      for (int k = 0; k < 2; ++k)
        asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(p[t][k]) : "r"(ptx::pack_bf16x2(e[2 * k], e[2 * k + 1])));
    }
  }
  // 16 rows' scores, [head][16]
  __device__ __forceinline__ void leave_scores(int t, float* out) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int g = (lane & 3) * 2 + (i & 1);
      if (g < G) out[g * 16 + (lane >> 2) + (i >> 1) * 8] = x[t][i];
    }
  }
  // lanes of a row nobody sees load 16 bytes of zeros instead: zero times an infinity is not zero
  __device__ __forceinline__ void value(const WarpPlace& w, uint32_t stage, unsigned visible, uint32_t zeros) {
    // A = 16 columns x 16 keys: matrices (columns 0-7, keys 0-7), (8-15, 0-7), (0-7, 8-15), (8-15, 8-15), each stored by keys
    const int r = (lane >> 4) * 8 + (lane & 7), piece = (lane >> 3) & 1;
    uint32_t a[2][KC][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t seen = (visible >> (16 * t + r)) & 1u, base = seen ? w.base[t] + stage : zeros;
#pragma unroll
      for (int c = 0; c < KC; ++c) ldm_x4_trans(a[t][c], base + seen * box_at(w.box_rows, w.r0[t] + r, c * 2 + piece));
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < KC; ++c) mma_16816(o[c], a[t][c], p[t][0], p[t][1]);
  }
  // To shared memory: outputs [G][kStateRow], maxima and sums [G].
  __device__ __forceinline__ void leave(float* out, float* ms, float* ls) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) l[h] += __shfl_xor_sync(0xffffffffu, l[h], off);
      const int g = (lane & 3) * 2 + h;
      if (g >= G) continue;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        out[g * state_row(D) + c * 16 + (lane >> 2)] = o[c][h];
        out[g * state_row(D) + c * 16 + (lane >> 2) + 8] = o[c][2 + h];
      }
      if (lane < 4) { ms[g] = m[h]; ls[g] = l[h]; }
    }
  }
};

// fp32: a lane is a row for the scores and owns D / 32 columns of the outputs.  GT: the group, up to a power of two (the
// heads behind it repeat the last one and are not written).
template <int D, int GT>
struct WarpRows<float, D, GT> {
  static constexpr int E = D / 32;
  const float* q;            // shared memory [heads][D]
  float o[GT][E], m[GT], l[GT], x[GT], p[GT];
  int lane, G;

  __device__ __forceinline__ void begin(const float* queries, int heads) {
    lane = threadIdx.x & 31;
    G = heads;
    q = queries;
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      m[g] = -INFINITY;
      l[g] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[g][e] = 0.f;
    }
  }
  __device__ __forceinline__ void score(const WarpPlace& w, uint32_t stage, unsigned visible, float scale_log2e) {
    const uint32_t base = (lane < 16 ? w.base[0] : w.base[1]) + stage;
    const int row = (lane < 16 ? w.r0[0] : w.r0[1]) + (lane & 15);
    float s[GT], s2[GT];                   // two chains each
#pragma unroll
    for (int g = 0; g < GT; ++g) s[g] = s2[g] = 0.f;
#pragma unroll (GT <= 2 ? 8 : 4)
    for (int c = 0; c < D / 4; ++c) {
      float4 k;
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(k.x), "=f"(k.y), "=f"(k.z), "=f"(k.w) : "r"(base + box_at(w.box_rows, row, c)));
#pragma unroll
      for (int g = 0; g < GT; ++g) {
        const float4 v = *reinterpret_cast<const float4*>(q + min(g, G - 1) * D + c * 4);
        s[g] = fmaf(v.y, k.y, fmaf(v.x, k.x, s[g]));
        s2[g] = fmaf(v.w, k.w, fmaf(v.z, k.z, s2[g]));
      }
    }
    bool grew = false;
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      x[g] = (visible >> lane) & 1u ? (s[g] + s2[g]) * scale_log2e : -INFINITY;
      grew |= x[g] > m[g] + kGrow;
    }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int g = 0; g < GT; ++g) {
        float top = x[g];
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        if (top > m[g] + kGrow) {
          const float alpha = exp2f(m[g] - top);
          l[g] *= alpha;
#pragma unroll
          for (int e = 0; e < E; ++e) o[g][e] *= alpha;
          m[g] = top;
        }
      }
    }
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      p[g] = exp2f(x[g] - (m[g] == -INFINITY ? 0.f : m[g]));
      l[g] += p[g];
    }
  }
  __device__ __forceinline__ void leave_scores(int t, float* out) const {
    if (lane >> 4 != t) return;
#pragma unroll
    for (int g = 0; g < GT; ++g)
      if (g < G) out[g * 16 + (lane & 15)] = x[g];
  }
  __device__ __forceinline__ void value(const WarpPlace& w, uint32_t stage, unsigned visible, uint32_t zeros) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll 8
      for (int r = 0; r < 16; ++r) {
        // a row nobody sees has weight 0; its values are not read
        float v[E];
        const uint32_t seen = (visible >> (16 * t + r)) & 1u;
        const uint32_t from = w.base[t] + stage + box_at(w.box_rows, w.r0[t] + r, E == 4 ? lane : lane >> 1) + (E == 4 ? 0 : (lane & 1) * 8);
        const uint32_t at = zeros + seen * (from - zeros);
        if constexpr (E == 4)
          asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(at));
        else
          asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(at));
#pragma unroll
        for (int g = 0; g < GT; ++g) {
          const float wt = __shfl_sync(0xffffffffu, p[g], 16 * t + r);
#pragma unroll
          for (int e = 0; e < E; ++e) o[g][e] = fmaf(wt, v[e], o[g][e]);
        }
      }
  }
  __device__ __forceinline__ void leave(float* out, float* ms, float* ls) {
#pragma unroll
    for (int g = 0; g < GT; ++g) {
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) l[g] += __shfl_xor_sync(0xffffffffu, l[g], off);
      if (g >= G) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) out[g * state_row(D) + lane * E + e] = o[g][e];
      if (lane == 0) { ms[g] = m[g]; ls[g] = l[g]; }
    }
  }
};

constexpr int kJoinAhead = 8;        // partial results whose outputs are on their way together

// One warp merges the partial results of a unit's head in order: `parts` of them from `slot` on.
template <typename T, int D>
__device__ __forceinline__ void merge_head(const PagedWs& ws, int slot, int parts, int G, int g, T* out) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  float o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 1
  for (int c0 = 0; c0 < parts; c0 += kJoinAhead) {
    const int cn = min(kJoinAhead, parts - c0);
    const float2 ml = lane < cn ? __ldcg(ws.ml + size_t(slot + c0 + lane) * G + g) : make_float2(-INFINITY, 0.f);
    float v[kJoinAhead][E];
#pragma unroll
    for (int c = 0; c < kJoinAhead; ++c) {
      const float* a = ws.acc + (size_t(slot + c0 + min(c, cn - 1)) * G + g) * D + lane * E;
      if constexpr (E == 4) { const float4 t = __ldcg(reinterpret_cast<const float4*>(a)); v[c][0] = t.x; v[c][1] = t.y; v[c][2] = t.z; v[c][3] = t.w; }
      else { const float2 t = __ldcg(reinterpret_cast<const float2*>(a)); v[c][0] = t.x; v[c][1] = t.y; }
    }
    float mn = ml.x;
#pragma unroll
    for (int off = kJoinAhead / 2; off > 0; off >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, off));
    mn = fmaxf(m, __shfl_sync(0xffffffffu, mn, 0));
    const float from = mn == -INFINITY ? 0.f : mn, keep = exp2f(m - from), w = exp2f(ml.x - from);
    const float wl = w * ml.y;
    l *= keep;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= keep;
#pragma unroll
    for (int c = 0; c < kJoinAhead; ++c) {
      const float wc = __shfl_sync(0xffffffffu, w, c);
      l += __shfl_sync(0xffffffffu, wl, c);
      if (c < cn) {
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(wc, v[c][e], o[e]);
      }
    }
    m = mn;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] /= l;
  T* to = out + lane * E;
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float2*>(to + e) = make_float2(o[e], o[e + 1]);
    else *reinterpret_cast<uint32_t*>(to + e) = ptx::pack_bf16x2(o[e], o[e + 1]);
  }
}

template <typename T, int D, int GT>
__global__ void __launch_bounds__(PagedRing<T, D, GT>::kThreads, 1)
paged_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const T* __restrict__ q,
             const __grid_constant__ PagedArgs args, int G, int window, int n_sink, float scale_log2e, int64_t l2_keep, PagedWs ws, T* __restrict__ O) {
  using Ring = PagedRing<T, D, GT>;
  constexpr int kStages = Ring::kStages, kTeams = Ring::kTeams;
  extern __shared__ uint8_t paged_smem[];
  uint8_t* ring_buf = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(paged_smem) + 1023) & ~uintptr_t(1023));
  uint8_t* states = ring_buf + kStages * Ring::kStageBytes;
  uint8_t* query_buf = states + kTeams * Ring::kState;
  __shared__ BulkRing<kStages> ring;
  __shared__ PagedDeal<kTeams * kConsumers, kList> deal;
  __shared__ int abort_word, goes_on[kTeams], merge_here[kTeams];
  __shared__ __align__(16) uint32_t zeros[4];
  __shared__ uint64_t query_full[Ring::kQueries];
  __shared__ int page_buf[kPageBatches + 1][32];
  __shared__ float s_m[kTeams][kWarps][kMaxGroup], s_l[kTeams][kWarps][kMaxGroup];
  __shared__ int group_row[kStages][kGroups];      // a stage's pool rows / 16; -1: not a page of the pool
  volatile int* abort_flag = &abort_word;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < Ring::kQueries; ++i) ptx::mbar_init(&query_full[i], 1);
    ring.init(kTeams * kWarps);
    abort_word = 0;
    zeros[0] = zeros[1] = zeros[2] = zeros[3] = 0u;
    ptx::tma_prefetch_desc(&map_k);
    ptx::tma_prefetch_desc(&map_v);
  }
  pdl_wait();
  pdl_launch_dependents();
  // Looked at only where results are written: the load takes up to 2 us, and the first request does not wait for it.
  const int found_status = *reinterpret_cast<const volatile int*>(ws.status);
  const int share = int(blockIdx.x);
  const int box_rows = min(1 << args.page_shift, kPagedStep);      // rows of a box
  // A lane of the producer warp reads the page of one group of 16 rows: of steps 0 .. 3 of a batch, group lane % 8.  Pages
  // come asynchronously, kPageBatches batches ahead: a trip to memory takes 2 to 3 us while everybody streams, as
  // long as two steps.
  int ahead_i = 0, ahead_s = 0;
  auto request_pages = [&](int k, int rank0, int here) {
    int* to = &page_buf[k % (kPageBatches + 1)][lane];
    bool there = false;
    const int32_t* from = args.table;
    if (ahead_i < here) {
      const PagedPiece& p = deal.at(rank0, ahead_i);
      if (ahead_s + (lane >> 3) < p.n) {
        const PagedSpan span(p.len, window, n_sink);
        const int slot = span.slot0(p.s0 + ahead_s + (lane >> 3)) + (lane & 7) * 16;
        there = span.any_visible(slot & ~(box_rows - 1), box_rows);
        from += size_t(p.u) * args.max_pages + (slot >> args.page_shift);
      }
      ahead_s += 4;
      if (ahead_s >= p.n) { ahead_s = 0; ++ahead_i; }
    }
    if (there) cp_async_4(to, from);
    else *to = -1;
    cp_async_group();
  };
  // The rows of all units are held in memory that has another use later: of 512 units the teams' states, of more the ring, which
  // takes a fence (0.3 us of a short call).
  static_assert(kTeams * Ring::kState >= (512 + 512 / 32) * 4, "rows of 512 units");
  const bool few = args.n_units <= 512, hold = args.n_units + (args.n_units >> 5) <= kStages * Ring::kStageBytes / 4;
  typename PagedDeal<kTeams * kConsumers, kList>::Mine my;
  const PagedCut cut = deal.start(args, window, n_sink, share, my, hold ? reinterpret_cast<int*>(few ? states : ring_buf) : nullptr, hold && !few);
  const int n_pieces = deal.n_pieces();
  if (ws.steps && tid == 0) ws.records[share] = deal.record;       // for the second kernel
  int n = 0;                                                       // stages handed over so far
  bool ok = true;
  for (int rank0 = 0; rank0 < n_pieces; rank0 += kList) {
    deal.round(args, window, n_sink, my, cut, share, rank0);
    const int here = min(kList, n_pieces - rank0);
    if (warp == kTeams * kWarps) {
      // ------------------------------------------------------------- producer
      // The next call reads these rows again, from where they are: of every 64 runs of 128 pool rows (bit-reversed, so
      // that every share holds as many) as many as fit kL2Share of the L2 ask to stay, the others to go first, so
      // that code, states, tables and partial results stay as well.
      const uint64_t stays = ptx::l2_policy_evict_last(), streams = ptx::l2_policy_evict_first();
      const int keep = int(min(int64_t(64), l2_keep / max(1, cut.total - kPagedLead)));
      int batch = 0;
      ahead_i = ahead_s = 0;
      for (int k = 0; k < 2; ++k) request_pages(k, rank0, here);
      for (int i = 0; i < here && ok; ++i) {
        const PagedPiece piece = deal.at(rank0, i);
        const PagedSpan span(piece.len, window, n_sink);
        if (lane == 0) {       // the piece that had the place has been begun by all consumers: they released a stage of it
          const int k = (rank0 + i) % Ring::kQueries;
          const uint32_t bytes = uint32_t(G) * D * sizeof(T);
          ptx::mbar_arrive_expect_tx(&query_full[k], bytes);
          bulk_copy_g2s(query_buf + k * Ring::kQueryBytes, q + size_t(piece.u) * G * D, bytes, &query_full[k]);
        }
        for (int s = 0; s < piece.n && ok; s += 4) {
          if (batch == 0) {
            cp_async_pending<1>();                        // the others can wait until the first boxes are on their way
          } else {
            for (int k = batch == 1 ? 2 : batch + kPageBatches - 1; k < batch + kPageBatches; ++k) request_pages(k, rank0, here);
            cp_async_pending<kPageBatches - 1>();
          }
          const int page = page_buf[batch % (kPageBatches + 1)][lane];   // this lane's own request
          ++batch;
          for (int b = 0; b < 4 && s + b < piece.n && ok; ++b) {
            const int mine = __shfl_sync(0xffffffffu, page, b * 8 + (lane & 7));
            const int slot = span.slot0(piece.s0 + s + b) + (lane & 7) * 16;
            const bool good = unsigned(mine) < unsigned(args.n_pages);
            const bool wanted = lane < 8 && span.any_visible(slot & ~(box_rows - 1), box_rows);
            if (wanted && !good) report_bounds_ws(ws.status, kBoundsCacheRow, mine);
            const int row = (mine << args.page_shift) + (slot & ((1 << args.page_shift) - 1));
            const bool box = wanted && good && (slot & (box_rows - 1)) == 0;
            const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, box)) * box_rows * 128 * Ring::kBoxes;
            if (ws.steps) {
              PagedStepRecord* to = ws.steps + piece.step + piece.s0 + s + b;
              if (lane < 8) to->group[lane] = make_int2(wanted && good ? row >> 4 : -1, int(span.visible16(slot)));
              if (lane == 8) *reinterpret_cast<int2*>(&to->slot) = make_int2(piece.slot, piece.parts);
            }
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
                ptx::tma_load_3d_hint(ring_buf + stage * Ring::kStageBytes + lane * 16 * 128 * Ring::kBoxes, kv ? &map_v : &map_k, 0, row, 0,
                                      &ring.full[stage], (int(__brev(unsigned(row >> 7)) >> 26) < keep) ? stays : streams);
            }
          }
        }
      }
    } else {
      // ------------------------------------------------------------- consumers
      const int team = warp / kWarps, tw = warp % kWarps;
      WarpRows<T, D, GT> rows;
      WarpPlace place;
      place.box_rows = box_rows;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int r = tw * kWarpRows + t * 16;
        place.base[t] = ptx::smem_u32(ring_buf) + uint32_t(r & ~(box_rows - 1)) * 128u * Ring::kBoxes;
        place.r0[t] = r & (box_rows - 1);
      }
      const uint32_t zero_addr = ptx::smem_u32(zeros);
      float* state = reinterpret_cast<float*>(states + team * Ring::kState);
      for (int i = 0; i < here; ++i) {
        const PagedPiece piece = deal.at(rank0, i);
        if (kTeams > 1 && ((rank0 + i) & 1) != team) {
          // The other team's: its stages are waited for and released like one's own.  A barrier tells only whether its
          // last phase is over, so nobody may be further ahead or behind than the ring is long.
          for (int s = 0; s < 2 * piece.n; ++s, ++n) {
            if (ok) ok = __all_sync(0xffffffffu, ring.wait_full(n, abort_flag));
            if (lane == 0) ring.release(n);
          }
          continue;
        }
        const PagedSpan span(piece.len, window, n_sink);
        const int qk = (rank0 + i) % Ring::kQueries;
        if (ok) ok = __all_sync(0xffffffffu, ptx::mbar_wait(&query_full[qk], uint32_t((rank0 + i) / Ring::kQueries) & 1u, abort_flag));
        rows.begin(reinterpret_cast<const T*>(query_buf + qk * Ring::kQueryBytes), G);
        for (int s = 0; s < piece.n; ++s) {
          const int slot = span.slot0(piece.s0 + s) + tw * kWarpRows;
          unsigned visible = span.visible16(slot) | span.visible16(slot + 16) << 16;
          if (ok) ok = __all_sync(0xffffffffu, ring.wait_full(n, abort_flag));
          const int at0 = ok ? group_row[n % kStages][tw * 2] : -1, at1 = ok ? group_row[n % kStages][tw * 2 + 1] : -1;
          if (at0 < 0) visible &= 0xffff0000u;
          if (at1 < 0) visible &= 0xffffu;
          if (visible) {
            rows.score(place, (n % kStages) * Ring::kStageBytes, visible, scale_log2e);
            if (ws.score) {
              if (at0 >= 0) rows.leave_scores(0, ws.score + size_t(at0) * G * 16);
              if (at1 >= 0) rows.leave_scores(1, ws.score + size_t(at1) * G * 16);
            }
          }
          __syncwarp();
          if (lane == 0) ring.release(n);
          ++n;
          if (ok) ok = __all_sync(0xffffffffu, ring.wait_full(n, abort_flag));
          if (ok && visible) rows.value(place, (n % kStages) * Ring::kStageBytes, visible, zero_addr);
          __syncwarp();
          if (lane == 0) ring.release(n);
          ++n;
        }
        // ----------------------------------------------------------- the warps' states become the piece's
        rows.leave(state + tw * GT * state_row(D), s_m[team][tw], s_l[team][tw]);
        if (team_agrees(tid % kConsumers == 0, &goes_on[team], [&] { return !*abort_flag && !stops_call(found_status); },
                        [&] { team_sync(team); })) {
          const size_t at = size_t(share + piece.u) * G;
          for (int j = tid % kConsumers * 4; j < G * D; j += kConsumers * 4) {
            const int g = j / D, d = j - g * D;
            float ms[kWarps], M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) M = fmaxf(M, ms[w] = s_m[team][w][g]);
            const float from = M == -INFINITY ? 0.f : M;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            float l = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
              const float wt = exp2f(ms[w] - from);
              const float4 v = *reinterpret_cast<const float4*>(state + (w * GT + g) * state_row(D) + d);
              acc.x = fmaf(v.x, wt, acc.x);
              acc.y = fmaf(v.y, wt, acc.y);
              acc.z = fmaf(v.z, wt, acc.z);
              acc.w = fmaf(v.w, wt, acc.w);
              l = fmaf(s_l[team][w][g], wt, l);
            }
            if (piece.parts == 0) {
              const float inv = 1.f / l;
              T* out = O + size_t(piece.u) * G * D + j;
              if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(out) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
              else *reinterpret_cast<uint2*>(out) = make_uint2(ptx::pack_bf16x2(acc.x * inv, acc.y * inv), ptx::pack_bf16x2(acc.z * inv, acc.w * inv));
            } else {
              *reinterpret_cast<float4*>(ws.acc + at * D + j) = acc;
            }
            if (d == 0) ws.ml[at + g] = make_float2(M, l);
          }
          if (piece.parts > 0 && !ws.steps) {
            // whoever brings the unit's last partial result merges them
            team_sync(team);
            if (tid % kConsumers == 0) {
              __threadfence();
              int* ticket = ws.tickets + (piece.slot - piece.u);
              const bool all = atomicAdd(ticket, 1) == piece.parts - 1;
              if (all) *ticket = 0;                         // for the next call
              __threadfence();
              merge_here[team] = all;
            }
            team_sync(team);
            if (merge_here[team])
              for (int g = tw; g < G; g += kWarps) merge_head<T, D>(ws, piece.slot, piece.parts, G, g, O + (size_t(piece.u) * G + g) * D);
          }
        }
        team_sync(team);                        // the states are written over by the next piece
      }
    }
  }
  if (warp < kTeams * kWarps && !stops_call(found_status)) {
    // nobody's pieces: units without a visible slot give zeros
    constexpr int kDealers = kTeams * kConsumers;
    for (int u = share * kDealers + tid; u < args.n_units; u += int(gridDim.x) * kDealers)
      if (PagedSpan(u == share * kDealers + tid ? my.tail : deal.rows_of(args, nullptr, u), window, n_sink).n == 0)
        for (int j = 0; j < G * D; j += 16 / int(sizeof(T))) *reinterpret_cast<uint4*>(O + size_t(u) * G * D + j) = make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  if (*abort_flag) {
    if (tid == 0) atomicCAS(ws.status, kStatusBounds, kStatusTimeout);
    ptx::abort_teardown(ws.status, tid);
  }
}

// ------------------------------------------------------------------ weights, and the merge of the partial results beside them
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;
constexpr int kWeightBlocks = 3;     // per SM

// For calls that accumulate weights.  The first weight_blocks blocks: a warp per step of 128 slots turns its scores into
// weights.  The others: one warp per (share, head) merges the partial results of the unit that begins there and runs on.  All
// loads that do not depend on one another are issued together: the kernel is a chain of trips to memory.
template <typename T, int D, int GT>
__global__ void __launch_bounds__(kJoinThreads, kWeightBlocks)
paged_join_kernel(int G, int n_shares, int weight_blocks, PagedWs ws, float* __restrict__ mass, T* __restrict__ O) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  pdl_launch_dependents();
  const int found_status = __ldcg(ws.status);
  auto stopped = [&] { return __any_sync(0xffffffffu, stops_call(found_status)); };   // what follows needs whole warps
  if (int(blockIdx.x) >= weight_blocks) {
    const int at = (int(blockIdx.x) - weight_blocks) * kJoinWarps + warp, share = at / G, g = at - share * G;
    if (share >= n_shares) return;
    const int4 rec = __ldcg(reinterpret_cast<const int4*>(ws.records) + share);
    if (stopped()) return;
    if (rec.z > 0) merge_head<T, D>(ws, rec.y, rec.z, G, g, O + (size_t(rec.x) * G + g) * D);
    return;
  }
  // ---- weights
  const int warps = weight_blocks * kJoinWarps;
  const int total = __ldcg(&ws.records[0].steps);
  if (stopped()) return;
  const float inv_g = 1.f / float(G);
  int2 where, next_where, group[4];
  auto fetch = [&](int step) {               // the record of the step after this one is on its way during this one
    const PagedStepRecord* rec = ws.steps + step;
    next_where = __ldcg(reinterpret_cast<const int2*>(&rec->slot));
#pragma unroll
    for (int i = 0; i < 4; ++i) group[i] = __ldcg(&rec->group[i * 2 + (lane >> 4)]);
  };
  int step = int(blockIdx.x) * kJoinWarps + warp;
  if (step < total) fetch(step);
  for (; step < total; step += warps) {
    where = next_where;
    int row[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) row[i] = group[i].x >= 0 && ((group[i].y >> (lane & 15)) & 1) ? group[i].x * 16 + (lane & 15) : -1;
    if (step + warps < total) fetch(step + warps);
    // the row sums: log2 of the sum over the unit's partial results, head by head
    float lse[GT];
    const int parts = max(1, where.y);
    float x[4][GT], sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum[i] = row[i] >= 0 ? mass[row[i]] : 0.f;
#pragma unroll
      for (int g = 0; g < GT; ++g)
        x[i][g] = g < G && row[i] >= 0 ? __ldcg(ws.score + (size_t(row[i] >> 4) * G + g) * 16 + (row[i] & 15)) : 0.f;
    }
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      lse[g] = 0.f;
      if (g >= G) continue;
      float m = -INFINITY, l = 0.f;
      for (int c = lane; c < parts; c += 32) {
        const float2 ml = __ldcg(ws.ml + size_t(where.x + c) * G + g);
        const float mn = fmaxf(m, ml.x), from = mn == -INFINITY ? 0.f : mn;
        l = l * exp2f(m - from) + ml.y * exp2f(ml.x - from);
        m = mn;
      }
      if (parts > 1) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
          const float mo = __shfl_xor_sync(0xffffffffu, m, off), lo2 = __shfl_xor_sync(0xffffffffu, l, off);
          const float mn = fmaxf(m, mo), from = mn == -INFINITY ? 0.f : mn;
          l = l * exp2f(m - from) + lo2 * exp2f(mo - from);
          m = mn;
        }
      }
      lse[g] = __shfl_sync(0xffffffffu, m + log2f(l), 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (row[i] < 0) continue;
      float w = 0.f;
#pragma unroll
      for (int g = 0; g < GT; ++g)
        if (g < G) w += exp2f(x[i][g] - lse[g]);
      mass[row[i]] = sum[i] + w * inv_g;
    }
  }
}

// The pool as [column block][row][128 bytes]: boxes of all columns of up to 128 rows.
template <typename T, int D>
bool pool_map(CUtensorMap* out, const void* base, const tca_paged_desc* c) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  constexpr int kCols = 128 / int(sizeof(T));
  cuuint64_t dims[3] = {cuuint64_t(kCols), cuuint64_t(c->n_pages) * c->page_size, cuuint64_t(PagedRing<T, D, 8>::kBoxes)};
  cuuint64_t strides[2] = {cuuint64_t(D) * sizeof(T), 128};
  cuuint32_t box[3] = {cuuint32_t(kCols), cuuint32_t(c->page_size < kPagedStep ? c->page_size : kPagedStep),
                       cuuint32_t(PagedRing<T, D, 8>::kBoxes)};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(out, sizeof(T) == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<void*>(base), dims,
            strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D, int GT>
int launch_paged(const tca_params* prm, const void* q, const tca_paged_desc* c, int n_sink, bool weights, void* O, const PagedWs& ws,
                 cudaStream_t s) {
  using Ring = PagedRing<T, D, GT>;
  CUtensorMap mk, mv;
  if (!pool_map<T, D>(&mk, c->k, c) || !pool_map<T, D>(&mv, c->v, c)) return TCA_ERR_CUDA;
  const int G = prm->n_q_heads / prm->n_kv_heads;
  const PagedArgs args = paged_args(c);
  constexpr auto kern = paged_kernel<T, D, GT>;
  if (allow_smem<kern>(Ring::kSmemBytes) != TCA_OK) return TCA_ERR_CUDA;
  const int st = launch_pdl(kern, dim3(unsigned(sm_count())), dim3(Ring::kThreads), size_t(Ring::kSmemBytes), s, mk, mv, static_cast<const T*>(q),
                            args, G, prm->window, n_sink, prm->sm_scale * kLog2e, int64_t(64 * kL2Share * double(l2_bytes()) / (2 * Ring::kStageBytes)), ws,
                            static_cast<T*>(O));
  if (st != TCA_OK || !weights) return st;
  const int merge_blocks = (sm_count() * G + kJoinWarps - 1) / kJoinWarps;
  const int weight_blocks = kWeightBlocks * sm_count();
  return launch_pdl(paged_join_kernel<T, D, (GT > 4 ? 8 : 4)>, dim3(unsigned(merge_blocks + weight_blocks)), dim3(kJoinThreads),
                    size_t(0), s, G, sm_count(), weight_blocks, ws, c->mass, static_cast<T*>(O));
}

template <int D>
int launch_paged_f32(const tca_params* prm, const void* q, const tca_paged_desc* c, int n_sink, bool weights, void* O, const PagedWs& ws,
                     cudaStream_t s) {
  const int G = prm->n_q_heads / prm->n_kv_heads;
  if (G == 1) return launch_paged<float, D, 1>(prm, q, c, n_sink, weights, O, ws, s);
  if (G == 2) return launch_paged<float, D, 2>(prm, q, c, n_sink, weights, O, ws, s);
  if (G <= 4) return launch_paged<float, D, 4>(prm, q, c, n_sink, weights, O, ws, s);
  return launch_paged<float, D, 8>(prm, q, c, n_sink, weights, O, ws, s);
}

}  // namespace
}  // namespace tca

using namespace tca;

extern "C" size_t tca_attn_paged_workspace_bytes(const tca_params* prm, const tca_paged_desc* c, int32_t accumulate) {
  if (check_paged(prm, c) != TCA_OK) return 0;
  return paged_ws_layout(prm, c, accumulate != 0, nullptr).bytes;
}

extern "C" int tca_attn_paged(const tca_params* prm, const void* q, const tca_paged_desc* c, int32_t n_sink, int32_t accumulate, void* O,
                              void* ws, size_t ws_bytes, void* stream) {
  const int st = check_paged(prm, c);
  if (st != TCA_OK) return st;
  TCA_CHECK_ARG(q && O && ws && n_sink >= 0);
  TCA_CHECK_ARG(aligned(q, 16) && aligned(O, 16) && aligned(ws, 256));
  if (prm->window < 1) return TCA_ERR_UNSUPPORTED;
  const PagedWs lay = paged_ws_layout(prm, c, accumulate != 0, ws);
  if (ws_bytes < lay.bytes) return TCA_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool w = accumulate != 0;
  if (prm->dtype == TCA_F32)
    return prm->head_dim == 128 ? launch_paged_f32<128>(prm, q, c, n_sink, w, O, lay, s) : launch_paged_f32<64>(prm, q, c, n_sink, w, O, lay, s);
  const bool wide = prm->n_q_heads > 4 * prm->n_kv_heads;
#define TCA_PAGED(D) (wide ? launch_paged<__nv_bfloat16, D, 8>(prm, q, c, n_sink, w, O, lay, s) : launch_paged<__nv_bfloat16, D, 4>(prm, q, c, n_sink, w, O, lay, s))
  return prm->head_dim == 128 ? TCA_PAGED(128) : TCA_PAGED(64);
#undef TCA_PAGED
}

extern "C" int tca_paged_status(const tca_paged_desc* c, void* stream, int64_t* detail) {
  TCA_CHECK_ARG(c && c->state && c->n_units >= 1 && c->n_units <= 65535);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  constexpr int kUnits = 1024;             // a part of the state at a time: no allocation
  int32_t st[kUnits * TCA_PG_STATE_WORDS];
  for (int64_t u0 = 0; u0 < c->n_units; u0 += kUnits) {
    const int64_t n = c->n_units - u0 < kUnits ? c->n_units - u0 : kUnits;
    TCA_CHECK_CUDA(cudaMemcpyAsync(st, c->state + u0 * TCA_PG_STATE_WORDS, size_t(n) * TCA_PG_STATE_WORDS * sizeof(int32_t),
                                   cudaMemcpyDeviceToHost, s));
    TCA_CHECK_CUDA(cudaStreamSynchronize(s));
    for (int64_t u = 0; u < n; ++u) {
      const int32_t which = st[u * TCA_PG_STATE_WORDS + TCA_PG_CHECK];
      if (which == 0) continue;
      if (detail) { detail[0] = u0 + u; detail[1] = which; }
      return TCA_ERR_BOUNDS;
    }
  }
  return TCA_OK;
}
