// tca_cache_accept: the accepted path of a drafted tree becomes ordinary tokens of the cache, exactly as
// one tca_cache_append per token would make them (Section 4.2, "Online Token Selection in Decoding
// Stage"), compression of the blocks that leave the window included.  One CTA per unit.  The tokens up to
// the next compression are written together; a compression scores its block with the queries of the token
// that filled the ring, as appending that token would.  Without a compression a call is one launch of 3 us;
// 512 units of which 200 compress take 14 us, bound by the latencies of a compression (its steps take turns: scores
// 4 us, softmax and ranks 3, everything around them 4).
#include "compress.cuh"

namespace tca {
namespace {

// Accepted counts travel as kernel arguments: the host needs them for its mirror anyway.
// The sequences that compress come first: a CTA that does runs seven times as long as one that does not, and not
// all CTAs are resident at once (17 -> 15.5 us for 512 units).  Those that accept nothing have no CTA.
constexpr int kSeqPerLaunch = 1024;
struct AcceptCounts {
  uint8_t n[kSeqPerLaunch];      // 1 .. TCA_TREE_MAX
  uint16_t seq[kSeqPerLaunch];   // which of the launch's sequences
};

template <typename T>
__global__ void __launch_bounds__(kCompressThreads, 2)
cache_accept_kernel(const T* __restrict__ k_draft, const T* __restrict__ v_draft, const T* __restrict__ q_draft, int n_draft,
                    const int32_t* __restrict__ path, const __grid_constant__ AcceptCounts counts, int seq0,
                    T* __restrict__ Kc, T* __restrict__ Vc, int32_t* __restrict__ pos, int64_t* __restrict__ state,
                    int64_t tail_cap, int D, int G, int n_kv, int b, int window, double sm_scale) {
  pdl_wait();
  pdl_launch_dependents();
  const int nth = int(blockIdx.x) / n_kv, seq = seq0 + counts.seq[nth];
  const int n = counts.n[nth];
  const int tid = threadIdx.x;
  const int64_t u = int64_t(seq) * n_kv + int(blockIdx.x) % n_kv;
  int64_t* st = state + u * TCA_STATE_WORDS;
  __shared__ int s_path[TCA_TREE_MAX];
  const int64_t seg = st[TCA_ST_SEG_START], gcap = st[TCA_ST_GLOBAL_CAP];
  int64_t n_global = st[TCA_ST_N_GLOBAL], tail_head = st[TCA_ST_TAIL_HEAD], n_tail = st[TCA_ST_N_TAIL];
  const int64_t seq_len = st[TCA_ST_SEQ_LEN];
  const int t_keep = int(st[TCA_ST_T_KEEP]);
  const int64_t ring = seg + gcap;
  if (tid < n) {
    int t = path[int64_t(seq) * n_draft + tid];
    if constexpr (kDebugBounds) {
      if (t < 0 || t >= n_draft) report_bounds_state(st, kBoundsDraftIndex, t);
    }
    s_path[tid] = min(max(t, 0), n_draft - 1);   // never a row outside the drafted buffers
  }
  __syncthreads();   // also: every thread has read the state before it is updated
  const int64_t full = int64_t(window) + b;
  if constexpr (kDebugBounds) {
    if (tail_head < 0 || tail_head >= tail_cap || n_tail < 0 || n_tail >= full || full > tail_cap) {
      if (tid == 0) report_bounds_state(st, kBoundsRingSlot, tail_head);
      return;
    }
  }
  // The host has checked the room for the counts of its mirror.  A captured call that is replayed moves on without
  // the mirror, so the unit's own words decide whether the tokens go in, in every build.
  const int over = int(n_tail + n - full);         // < n; b is a power of two
  const int blocks = over >= 0 ? (over >> (31 - __clz(b))) + 1 : 0;
  if (n_global + int64_t(blocks) * t_keep > gcap) {
    if (tid == 0) report_bounds_state(st, kBoundsGlobalRegion, n_global);
    return;
  }
  const int shift = 31 - __clz(D * int(sizeof(T)) / 16);   // 16-byte pieces per row: a power of two
  for (int i0 = 0; i0 < n;) {
    const int cnt = int(min(int64_t(n - i0), full - n_tail));   // >= 1: the ring never stays full
    for (int i = tid; i < cnt << shift; i += kCompressThreads) {
      const int j = i >> shift, e = i & ((1 << shift) - 1);
      int64_t slot = tail_head + n_tail + j;   // < 2 tail_cap: the ring has room for a full one
      if (slot >= tail_cap) slot -= tail_cap;
      const int64_t src = ((u * n_draft + s_path[i0 + j]) << shift) + e, dst = ((ring + slot) << shift) + e;
      reinterpret_cast<uint4*>(Kc)[dst] = reinterpret_cast<const uint4*>(k_draft)[src];
      reinterpret_cast<uint4*>(Vc)[dst] = reinterpret_cast<const uint4*>(v_draft)[src];
      if (e == 0) pos[ring + slot] = int32_t(seq_len + i0 + j);
    }
    i0 += cnt;
    n_tail += cnt;
    if (n_tail >= full) {
      __syncthreads();   // the appended rows are visible to the CTA (they are in the block when w is small)
      compress_oldest_block(q_draft + (u * G * n_draft + s_path[i0 - 1]) * D, int64_t(n_draft) * D, Kc, Vc, pos, seg, ring,
                            n_global, tail_head, tail_cap, t_keep, D, G, b, sm_scale);
      __syncthreads();   // the moved rows have been read: their slots may be written again
      n_global += t_keep;
      tail_head += b;
      if (tail_head >= tail_cap) tail_head -= tail_cap;
      n_tail -= b;
    }
  }
  if (tid == 0) {
    st[TCA_ST_N_GLOBAL] = n_global;
    st[TCA_ST_TAIL_HEAD] = tail_head;
    st[TCA_ST_N_TAIL] = n_tail;
    st[TCA_ST_SEQ_LEN] = seq_len + n;
  }
}

template <typename T>
int launch_accept(const tca_params* prm, tca_cache_desc* c, const void* k, const void* v, const void* q, int n_draft,
                  const int32_t* path, const AcceptCounts& counts, int seq0, int n_seq, cudaStream_t s) {
  return launch_pdl(cache_accept_kernel<T>, dim3(unsigned(n_seq * prm->n_kv_heads)), dim3(kCompressThreads), size_t(0), s,
                    static_cast<const T*>(k), static_cast<const T*>(v), static_cast<const T*>(q), n_draft, path, counts,
                    seq0, static_cast<T*>(c->k), static_cast<T*>(c->v), c->pos, c->state, c->tail_cap, prm->head_dim,
                    prm->n_q_heads / prm->n_kv_heads, prm->n_kv_heads, prm->block, prm->window, double(prm->sm_scale));
}

}  // namespace
}  // namespace tca

using namespace tca;

extern "C" int tca_cache_accept(const tca_params* prm, tca_cache_desc* c, const void* k_draft, const void* v_draft,
                                const void* q_draft, int32_t n_draft, const int32_t* path, const int32_t* n_accept,
                                void* stream) {
  int st = check_params(prm);
  if (st != TCA_OK) return st;
  TCA_CHECK_ARG(c && k_draft && v_draft && q_draft && path && n_accept);
  TCA_CHECK_ARG(c->k && c->v && c->pos && c->state && c->global_cap && c->n_global && c->tail_head && c->n_tail &&
                c->seq_len && c->t_keep);
  TCA_CHECK_ARG(n_draft >= 1);
  if (n_draft > TCA_TREE_MAX) return TCA_ERR_UNSUPPORTED;
  TCA_CHECK_ARG(aligned(k_draft, 16) && aligned(v_draft, 16) && aligned(q_draft, 16) && aligned(path, 4));
  TCA_CHECK_ARG(aligned(c->k, 16) && aligned(c->v, 16));
  const int H = prm->n_kv_heads;
  const int64_t U = int64_t(prm->batch) * H;
  TCA_CHECK_ARG(c->n_units == U && U < (int64_t(1) << 31));
  const int64_t full = int64_t(prm->window) + prm->block;
  if (c->tail_cap < full) return TCA_ERR_CAPACITY;
  // a ring is compressed each time it reaches `full`; everything is checked before anything changes
  auto compressions = [&](int64_t u, int64_t n) {
    const int64_t over = c->n_tail[u] + n - full;
    return over >= 0 ? over / prm->block + 1 : int64_t(0);
  };
  for (int32_t s = 0; s < prm->batch; ++s) {
    TCA_CHECK_ARG(n_accept[s] >= 0 && n_accept[s] <= n_draft);
    for (int h = 0; h < H; ++h) {
      const int64_t u = int64_t(s) * H + h;
      TCA_CHECK_ARG(c->n_tail[u] >= 0 && c->n_tail[u] < full);
      if (c->n_global[u] + compressions(u, n_accept[s]) * c->t_keep[u] > c->global_cap[u]) return TCA_ERR_CAPACITY;
      TCA_CHECK_ARG(c->seq_len[u] + n_accept[s] < (int64_t(1) << 31));
    }
  }
  for (int32_t s0 = 0; s0 < prm->batch; s0 += kSeqPerLaunch) {
    AcceptCounts counts;
    const int n_seq = prm->batch - s0 < kSeqPerLaunch ? prm->batch - s0 : kSeqPerLaunch;
    int listed = 0;
    for (int pass = 0; pass < 2; ++pass)
      for (int i = 0; i < n_seq; ++i) {
        const int32_t n = n_accept[s0 + i];
        if (n == 0 || (compressions(int64_t(s0 + i) * H, n) > 0) != (pass == 0)) continue;
        counts.n[listed] = uint8_t(n);
        counts.seq[listed++] = uint16_t(i);
      }
    if (listed == 0) continue;
    cudaStream_t str = static_cast<cudaStream_t>(stream);
    st = prm->dtype == TCA_BF16
             ? launch_accept<__nv_bfloat16>(prm, c, k_draft, v_draft, q_draft, n_draft, path, counts, s0, listed, str)
             : launch_accept<float>(prm, c, k_draft, v_draft, q_draft, n_draft, path, counts, s0, listed, str);
    if (st != TCA_OK) return st;
    for (int i = 0; i < n_seq; ++i) {
      const int64_t n = n_accept[s0 + i];
      for (int h = 0; h < H; ++h) {
        const int64_t u = int64_t(s0 + i) * H + h;
        const int64_t k = compressions(u, n);
        c->n_global[u] += k * c->t_keep[u];
        if (k > 0) c->tail_head[u] = (c->tail_head[u] + k * prm->block) % c->tail_cap;
        c->n_tail[u] += n - k * prm->block;
        c->seq_len[u] += n;
      }
    }
  }
  return TCA_OK;
}
