// tca_paged_append: rows of packed prompts, or one new token per sequence, go to the end of paged sequences.  A copy,
// bound by memory for prompts and by latency for single tokens: 159 MB read and written in 31.6 us (5.0 TB/s, the
// launch and the lookups of lengths and pages among them), a token each for 64 sequences in 3.1 us.
#include <cstring>

#include "packed_common.cuh"
#include "paged_common.cuh"

namespace tca {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerCta = 128;
constexpr int kSeqPerLaunch = 256;       // places that travel as kernel arguments (4 KB)

struct AppendBuffers {
  const uint4 *K, *V;                    // views in 16-byte pieces
  PackedView kview, vview;
  const float* mass;                     // [n_kv_heads][rows], or null
  int64_t rows;
  uint4 *Kc, *Vc;
  int32_t* pos;
  float* mass_c;
  int shift;                             // log2 of a row's pieces
  int n_kv;
};

// One row per sequence: a warp per unit, which is alone with the unit's state.
struct AppendSlots {
  int32_t slot[kSeqPerLaunch];
};
__global__ void __launch_bounds__(kThreads)
append_step_kernel(const __grid_constant__ AppendBuffers b, const __grid_constant__ PagedArgs args, int seq0, int n_seq, bool placed,
                   const __grid_constant__ AppendSlots slots) {
  const int at = (int(blockIdx.x) * kThreads + int(threadIdx.x)) >> 5, lane = threadIdx.x & 31;
  const int i = at / b.n_kv, h = at - i * b.n_kv;
  pdl_wait();
  pdl_launch_dependents();
  if (i >= n_seq) return;
  const int u = (placed ? slots.slot[i] : seq0 + i) * b.n_kv + h;
  const int64_t row = seq0 + i;
  const uint4* ks = b.K + h * b.kview.head + row * b.kview.row;
  const uint4* vs = b.V + h * b.vview.head + row * b.vview.row;
  const int pieces = 1 << b.shift;
  const uint4 kv = lane < pieces ? ks[lane] : make_uint4(0, 0, 0, 0);
  const uint4 vv = lane < pieces ? vs[lane] : make_uint4(0, 0, 0, 0);
  int4* st = args.state + u;
  const int len = st->x, next = st->y;
  if (len < 0 || len >= args.max_pages << args.page_shift) {
    if (lane == 0) report_paged(st, kPagedNoRoom);
    return;
  }
  const int dst = paged_row(args, u, len);
  if (dst < 0) {
    if (lane == 0) report_paged(st, kPagedBadPage);
    return;
  }
  if (lane < pieces) {
    b.Kc[(int64_t(dst) << b.shift) + lane] = kv;
    b.Vc[(int64_t(dst) << b.shift) + lane] = vv;
  }
  if (lane == 0) {
    b.pos[dst] = next;
    b.mass_c[dst] = b.mass ? b.mass[h * b.rows + row] : 0.f;
    st->x = len + 1;
    st->y = next + 1;
  }
}

// Prompts: one CTA moves 128 rows of K and V of one sequence and KV head.  The CTAs of a unit all read its length before
// the last of them to arrive (a count in the state) moves it on.
struct AppendSeqs {
  int32_t row0[kSeqPerLaunch], len[kSeqPerLaunch], slot[kSeqPerLaunch];
  int32_t first_cta[kSeqPerLaunch + 1];
  int n;
};
constexpr unsigned kFailed = 1u << 30;   // of the count: a CTA found no page for a row

__global__ void __launch_bounds__(kThreads)
append_rows_kernel(const __grid_constant__ AppendBuffers b, const __grid_constant__ PagedArgs args, const __grid_constant__ AppendSeqs seqs) {
  __shared__ int dst[kRowsPerCta];
  pdl_wait();
  pdl_launch_dependents();
  const int h = int(blockIdx.y), cta = int(blockIdx.x), tid = int(threadIdx.x);
  int lo = 0, hi = seqs.n;                // the last sequence whose first CTA is <= cta
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (seqs.first_cta[mid] <= cta) lo = mid; else hi = mid;
  }
  const int n_new = seqs.len[lo], u = seqs.slot[lo] * b.n_kv + h;
  const int r0 = (cta - seqs.first_cta[lo]) * kRowsPerCta, n = min(kRowsPerCta, n_new - r0);
  const int64_t row = int64_t(seqs.row0[lo]) + r0;
  const uint4* ks = b.K + h * b.kview.head + row * b.kview.row;
  const uint4* vs = b.V + h * b.vview.head + row * b.vview.row;
  uint4 kv[4], vv[4];
  auto fetch = [&](int p0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = p0 + i * kThreads;
      if (p < (n << b.shift)) {
        const int r = p >> b.shift, c = p & ((1 << b.shift) - 1);
        kv[i] = __ldcs(ks + r * b.kview.row + c);
        vv[i] = __ldcs(vs + r * b.vview.row + c);
      }
    }
  };
  fetch(tid);                             // on its way while the length and the pages are looked up
  int4* st = args.state + u;
  const int len = st->x, next = st->y;
  if (len < 0 || int64_t(len) + n_new > int64_t(args.max_pages) << args.page_shift) {   // the same for all of the unit's CTAs
    if (r0 == 0 && tid == 0) report_paged(st, kPagedNoRoom);
    return;
  }
  bool bad = false;
  if (tid < n) {
    dst[tid] = paged_row(args, u, len + r0 + tid);
    bad = dst[tid] < 0;
  }
  bad = __syncthreads_or(bad);
  if (tid == 0) {
    unsigned* count = reinterpret_cast<unsigned*>(st) + TCA_PG_RESERVED;
    if (bad) {
      atomicOr(count, kFailed);
      report_paged(st, kPagedBadPage);
    }
    __threadfence();
    const unsigned before = atomicAdd(count, 1u);
    if ((before & ~kFailed) == unsigned(seqs.first_cta[lo + 1] - seqs.first_cta[lo] - 1)) {
      __threadfence();                    // the others' reads of the length come before what is written to it here
      if (!(before & kFailed)) {
        st->x = len + n_new;
        st->y = next + n_new;
      }
      *count = 0;
    }
  }
  for (int p0 = tid; p0 < (n << b.shift); p0 += 4 * kThreads) {
    if (p0 != tid) fetch(p0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = p0 + i * kThreads;
      if (p < (n << b.shift) && dst[p >> b.shift] >= 0) {
        const int64_t d = (int64_t(dst[p >> b.shift]) << b.shift) + (p & ((1 << b.shift) - 1));
        b.Kc[d] = kv[i];
        b.Vc[d] = vv[i];
      }
    }
  }
  if (tid < n && dst[tid] >= 0) {
    b.pos[dst[tid]] = next + r0 + tid;
    b.mass_c[dst[tid]] = b.mass ? b.mass[h * b.rows + row + tid] : 0.f;
  }
}

}  // namespace
}  // namespace tca

using namespace tca;

extern "C" int tca_paged_append(const tca_params* prm, const void* K, const void* V, int64_t rows, const int64_t* strides,
                                const int64_t* seq_start, const int32_t* slots, int32_t n_seq, const float* mass, tca_paged_desc* c,
                                void* stream) {
  int st = check_paged(prm, c);
  if (st != TCA_OK) return st;
  TCA_CHECK_ARG((K && V) || rows == 0);
  TCA_CHECK_ARG(rows >= 0 && rows < (int64_t(1) << 31) && n_seq >= 0 && n_seq <= prm->batch);
  TCA_CHECK_ARG(aligned(K, 16) && aligned(V, 16) && aligned(mass, 4));
  TCA_CHECK_ARG(seq_start || n_seq <= rows);
  const int H = prm->n_kv_heads;
  const int64_t unit = 16 / int64_t(elt_size(prm->dtype));
  int64_t sv[4];   // K head, K row, V head, V row strides in elements
  for (int i = 0; i < 4; ++i) {
    sv[i] = strides ? strides[i] : (i % 2 == 0 ? (rows > 0 ? rows : 1) * prm->head_dim : int64_t(prm->head_dim));
    TCA_CHECK_ARG(sv[i] >= prm->head_dim && sv[i] % unit == 0 && sv[i] < (int64_t(1) << 36));
  }
  for (int i = 0; i < n_seq && seq_start; ++i)
    TCA_CHECK_ARG(seq_start[i] >= 0 && seq_start[i + 1] >= seq_start[i] && seq_start[i + 1] <= rows);
  // two sequences cannot go to the same place: a bit per place, so many places at a time
  constexpr int kPlaces = 8192;
  for (int i = 0; i < n_seq && slots; ++i) TCA_CHECK_ARG(slots[i] >= 0 && slots[i] < prm->batch);
  for (int64_t p0 = 0; slots && p0 < prm->batch; p0 += kPlaces) {
    uint32_t taken[kPlaces / 32] = {};
    for (int i = 0; i < n_seq; ++i) {
      const int64_t p = slots[i] - p0;
      if (p < 0 || p >= kPlaces) continue;
      TCA_CHECK_ARG(!(taken[p / 32] >> (p % 32) & 1u));
      taken[p / 32] |= 1u << (p % 32);
    }
  }
  AppendBuffers b;
  b.K = static_cast<const uint4*>(K);
  b.V = static_cast<const uint4*>(V);
  b.kview = PackedView{sv[0] / unit, sv[1] / unit};
  b.vview = PackedView{sv[2] / unit, sv[3] / unit};
  b.mass = mass;
  b.rows = rows;
  b.Kc = static_cast<uint4*>(c->k);
  b.Vc = static_cast<uint4*>(c->v);
  b.pos = c->pos;
  b.mass_c = c->mass;
  b.n_kv = H;
  b.shift = 0;
  while ((16 << b.shift) < int64_t(prm->head_dim) * int64_t(elt_size(prm->dtype))) ++b.shift;
  const PagedArgs args = paged_args(c);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (!seq_start) {
    const int step = slots ? kSeqPerLaunch : n_seq;
    for (int i0 = 0; i0 < n_seq; i0 += step) {
      const int n = n_seq - i0 < step ? n_seq - i0 : step;
      AppendSlots a = {};
      if (slots) std::memcpy(a.slot, slots + i0, size_t(n) * sizeof(int32_t));
      const int64_t warps = int64_t(n) * H;
      st = launch_pdl(append_step_kernel, dim3(unsigned((warps * 32 + kThreads - 1) / kThreads)), dim3(kThreads), size_t(0), s, b, args, i0, n,
                      slots != nullptr, a);
      if (st != TCA_OK) return st;
    }
    return TCA_OK;
  }
  for (int i0 = 0; i0 < n_seq; i0 += kSeqPerLaunch) {
    AppendSeqs seqs;
    seqs.n = n_seq - i0 < kSeqPerLaunch ? n_seq - i0 : kSeqPerLaunch;
    int64_t ctas = 0;
    for (int i = 0; i < seqs.n; ++i) {
      const int64_t len = seq_start[i0 + i + 1] - seq_start[i0 + i];
      seqs.row0[i] = int32_t(seq_start[i0 + i]);
      seqs.len[i] = int32_t(len);
      seqs.slot[i] = slots ? slots[i0 + i] : i0 + i;
      seqs.first_cta[i] = int32_t(ctas);
      ctas += (len + kRowsPerCta - 1) / kRowsPerCta;
    }
    seqs.first_cta[seqs.n] = int32_t(ctas);
    if (ctas == 0) continue;
    st = launch_pdl(append_rows_kernel, dim3(unsigned(ctas), unsigned(H)), dim3(kThreads), size_t(0), s, b, args, seqs);
    if (st != TCA_OK) return st;
  }
  return TCA_OK;
}
