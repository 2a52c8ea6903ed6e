// tca_cache_load: packed prompts enter the retained cache with everything they hold (a 100 % budget):
// what tca_compact_kv does for a batch of one length and a selection, for prompts of different lengths
// and chosen places in the cache.  A copy, bound by memory: every retained row is read and written once.
// 592 MB (prompts of up to 32K tokens) take 92.3 us, 6.42 TB/s = 99 % of the measured copy bandwidth;
// 37.6 MB (a batch of chat prompts) 8.1 us, most of it from L2.
#include "packed_common.cuh"

namespace tca {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerCta = 128;
// Sequences per launch.  Their starts, lengths and slots travel as kernel arguments (the host knows
// them; no device copy to keep alive), which have room for 4 KB.
constexpr int kSeqPerLaunch = 96;

struct LoadSeqs {
  int64_t row0[kSeqPerLaunch];
  int32_t len[kSeqPerLaunch];
  int32_t slot[kSeqPerLaunch];
  int32_t first_cta[kSeqPerLaunch + 1];   // CTAs of all earlier sequences (per KV head)
  int n;
};

// One CTA moves 128 rows of K and of V of one sequence and KV head.  16-byte pieces, a row's pieces in
// adjacent lanes; eight loads in flight per thread before the first store.
__global__ void __launch_bounds__(kThreads)
load_kernel(const uint4* __restrict__ K, const uint4* __restrict__ V, const __grid_constant__ LoadSeqs seqs,
            PackedView kview, PackedView vview, int shift, int block, int window, uint4* __restrict__ Kc,
            uint4* __restrict__ Vc, int32_t* __restrict__ pos, int64_t* __restrict__ state, int64_t tail_cap) {
  pdl_wait();
  pdl_launch_dependents();
  const int n_kv = int(gridDim.y), h = int(blockIdx.y), cta = int(blockIdx.x);
  int lo = 0, hi = seqs.n;                // the last sequence whose first CTA is <= cta
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (seqs.first_cta[mid] <= cta) lo = mid; else hi = mid;
  }
  const int len = seqs.len[lo];
  const int64_t row0 = seqs.row0[lo];
  int64_t* st = state + (int64_t(seqs.slot[lo]) * n_kv + h) * TCA_STATE_WORDS;
  const int64_t seg = st[TCA_ST_SEG_START], gcap = st[TCA_ST_GLOBAL_CAP];
  const int n_glob = len > window ? (len - window) / block * block : 0;
  const int r0 = (cta - seqs.first_cta[lo]) * kRowsPerCta;
  if constexpr (kDebugBounds) {
    // the host checked its mirror of these words; the device words must agree
    if (n_glob > gcap || len - n_glob > tail_cap) {
      if (threadIdx.x == 0) report_bounds_state(st, kBoundsGlobalRegion, n_glob);
      return;
    }
  }
  if (r0 == 0 && threadIdx.x == 0) {
    st[TCA_ST_N_GLOBAL] = n_glob;
    st[TCA_ST_TAIL_HEAD] = 0;
    st[TCA_ST_N_TAIL] = len - n_glob;
    st[TCA_ST_SEQ_LEN] = len;
  }
  const int n = min(kRowsPerCta, len - r0);
  // cache row of prompt row r: the ring lies gcap rows behind the global region's start
  auto dst_row = [&](int r) { return r < n_glob ? seg + r : seg + gcap + (r - n_glob); };
  const uint4* ks = K + int64_t(h) * kview.head + (row0 + r0) * kview.row;   // views in 16-byte pieces here
  const uint4* vs = V + int64_t(h) * vview.head + (row0 + r0) * vview.row;
  for (int p0 = threadIdx.x; p0 < (n << shift); p0 += 4 * kThreads) {
    uint4 kv[4], vv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = p0 + i * kThreads;
      if (p < (n << shift)) {
        const int r = p >> shift, c = p & ((1 << shift) - 1);
        kv[i] = __ldcs(ks + r * kview.row + c);
        vv[i] = __ldcs(vs + r * vview.row + c);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = p0 + i * kThreads;
      if (p < (n << shift)) {
        const int r = p >> shift, c = p & ((1 << shift) - 1);
        const int64_t d = (dst_row(r0 + r) << shift) + c;
        Kc[d] = kv[i];
        Vc[d] = vv[i];
      }
    }
  }
  for (int r = threadIdx.x; r < n; r += kThreads) pos[dst_row(r0 + r)] = r0 + r;
}

}  // namespace
}  // namespace tca

using namespace tca;

extern "C" int tca_cache_load(const tca_params* prm, const void* K, const void* V, int64_t rows, const int64_t* strides,
                              const int64_t* seq_start, const int32_t* slots, int32_t n_seq, tca_cache_desc* c,
                              void* stream) {
  int st = check_params(prm);
  if (st != TCA_OK) return st;
  TCA_CHECK_ARG(((K && V) || rows == 0) && seq_start && c);   // no rows: nothing that K and V would point at
  TCA_CHECK_ARG(c->k && c->v && c->pos && c->state && c->seg_start && c->global_cap && c->n_global && c->tail_head &&
                c->n_tail && c->seq_len);
  TCA_CHECK_ARG(rows >= 0 && rows < (int64_t(1) << 31) && n_seq >= 0 && n_seq <= prm->batch);
  TCA_CHECK_ARG(aligned(K, 16) && aligned(V, 16) && aligned(c->k, 16) && aligned(c->v, 16));
  const int H = prm->n_kv_heads;
  TCA_CHECK_ARG(c->n_units == int64_t(prm->batch) * H && H <= 65535);
  const int64_t unit = 16 / int64_t(elt_size(prm->dtype));
  int64_t sv[4];   // K head, K row, V head, V row strides in elements
  for (int i = 0; i < 4; ++i) {
    sv[i] = strides ? strides[i] : (i % 2 == 0 ? (rows > 0 ? rows : 1) * prm->head_dim : int64_t(prm->head_dim));
    TCA_CHECK_ARG(sv[i] >= prm->head_dim && sv[i] % unit == 0 && sv[i] < (int64_t(1) << 36));
  }
  auto blocks_of = [&](int64_t len) { return num_blocks(prm, len) * prm->block; };
  // everything is checked before anything is launched or any mirror changes
  for (int i = 0; i < n_seq; ++i) {
    TCA_CHECK_ARG(seq_start[i] >= 0 && seq_start[i + 1] >= seq_start[i] && seq_start[i + 1] <= rows);
    const int64_t slot = slots ? slots[i] : i;
    TCA_CHECK_ARG(slot >= 0 && slot < prm->batch);
    const int64_t len = seq_start[i + 1] - seq_start[i], ng = blocks_of(len);
    for (int h = 0; h < H; ++h)
      if (ng > c->global_cap[slot * H + h] || len - ng > c->tail_cap) return TCA_ERR_CAPACITY;
  }
  // two prompts cannot share a place: a bit per place, so many places at a time
  constexpr int kPlaces = 8192;
  for (int64_t p0 = 0; slots && p0 < prm->batch; p0 += kPlaces) {
    uint32_t taken[kPlaces / 32] = {};
    for (int i = 0; i < n_seq; ++i) {
      const int64_t p = slots[i] - p0;
      if (p < 0 || p >= kPlaces) continue;
      TCA_CHECK_ARG(!(taken[p / 32] >> (p % 32) & 1u));
      taken[p / 32] |= 1u << (p % 32);
    }
  }
  const int pieces = int(prm->head_dim * elt_size(prm->dtype) / 16);
  int shift = 0;
  while ((1 << shift) < pieces) ++shift;
  const PackedView kview{sv[0] / unit, sv[1] / unit}, vview{sv[2] / unit, sv[3] / unit};
  for (int i0 = 0; i0 < n_seq; i0 += kSeqPerLaunch) {
    LoadSeqs seqs;
    seqs.n = n_seq - i0 < kSeqPerLaunch ? n_seq - i0 : kSeqPerLaunch;
    int64_t ctas = 0;
    for (int i = 0; i < seqs.n; ++i) {
      const int64_t len = seq_start[i0 + i + 1] - seq_start[i0 + i];
      seqs.row0[i] = seq_start[i0 + i];
      seqs.len[i] = int32_t(len);
      seqs.slot[i] = slots ? slots[i0 + i] : i0 + i;
      seqs.first_cta[i] = int32_t(ctas);
      ctas += len > 0 ? (len + kRowsPerCta - 1) / kRowsPerCta : 1;   // an empty prompt still sets the state words
    }
    seqs.first_cta[seqs.n] = int32_t(ctas);
    st = launch_pdl(load_kernel, dim3(unsigned(ctas), unsigned(H)), dim3(kThreads), size_t(0),
                    static_cast<cudaStream_t>(stream), static_cast<const uint4*>(K), static_cast<const uint4*>(V), seqs,
                    kview, vview, shift, prm->block, prm->window, static_cast<uint4*>(c->k), static_cast<uint4*>(c->v),
                    c->pos, c->state, c->tail_cap);
    if (st != TCA_OK) return st;
    for (int i = 0; i < seqs.n; ++i) {
      const int64_t len = seqs.len[i], ng = blocks_of(len);
      for (int h = 0; h < H; ++h) {
        const int64_t u = int64_t(seqs.slot[i]) * H + h;
        c->n_global[u] = ng;
        c->tail_head[u] = 0;
        c->n_tail[u] = len - ng;
        c->seq_len[u] = len;
      }
    }
  }
  return TCA_OK;
}
