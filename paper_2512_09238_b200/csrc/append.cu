// tca_cache_append: decode-time cache maintenance (Section 4.2, "Online Token Selection
// in Decoding Stage").  One CTA per unit: write the new key/value into the tail ring and,
// when the ring then holds window + block tokens, compress the block that leaves the
// window: score its b keys with the current query group (Eq. 5 restricted to the block,
// fp64), keep the top t_keep by the order the prefill uses, and move those
// rows to the end of the global region in ascending position.
#include "common.cuh"
#include "compress.cuh"

namespace tca {
namespace {

constexpr int kThreads = kCompressThreads;

template <typename T>
__global__ void __launch_bounds__(kThreads, 2)
cache_append_kernel(const T* __restrict__ k_new, const T* __restrict__ v_new, const T* __restrict__ q_cur,
                    T* __restrict__ Kc, T* __restrict__ Vc, int32_t* __restrict__ pos,
                    int64_t* __restrict__ state, int64_t tail_cap, int D, int G, int b, int window,
                    double sm_scale) {
  pdl_wait();                 // the previous step's kernels still read the cache and its state
  pdl_launch_dependents();
  const int u = blockIdx.x;
  const int tid = threadIdx.x;
  int64_t* st = state + size_t(u) * TCA_STATE_WORDS;
  // the new row is requested together with the state words (one trip to memory instead of two);
  // head_dim <= 128 < kThreads, so a thread holds at most one element of it
  T k_val = T(), v_val = T();
  if (tid < D) {
    k_val = k_new[size_t(u) * D + tid];
    v_val = v_new[size_t(u) * D + tid];
  }
  const int64_t seg = st[TCA_ST_SEG_START], gcap = st[TCA_ST_GLOBAL_CAP];
  const int64_t n_global = st[TCA_ST_N_GLOBAL], tail_head = st[TCA_ST_TAIL_HEAD];
  const int64_t n_tail = st[TCA_ST_N_TAIL], seq_len = st[TCA_ST_SEQ_LEN];
  const int t_keep = int(st[TCA_ST_T_KEEP]);
  const int64_t ring = seg + gcap;
  __syncthreads();  // every thread has read the state before anyone updates it

  if constexpr (kDebugBounds) {
    // the state words this kernel indexes with: ring position and fill, and room for a kept block
    const bool bad_ring = tail_head < 0 || tail_head >= tail_cap || n_tail < 0 || n_tail >= tail_cap;
    const bool bad_room = (n_tail + 1 >= int64_t(window) + b) && (t_keep < 0 || t_keep > b);
    if (bad_ring || bad_room) {
      if (tid == 0) report_bounds_state(st, bad_ring ? kBoundsRingSlot : kBoundsGlobalRegion, bad_ring ? tail_head : n_global);
      return;
    }
  }
  // ---- append
  {
    const int64_t slot = (tail_head + n_tail) % tail_cap;
    if (tid < D) {
      Kc[(ring + slot) * D + tid] = k_val;
      Vc[(ring + slot) * D + tid] = v_val;
    }
    if (tid == 0) pos[ring + slot] = int32_t(seq_len);
  }
  const int64_t n_tail1 = n_tail + 1;
  const bool compress = n_tail1 >= int64_t(window) + b;
  if (!compress) {
    if (tid == 0) {
      st[TCA_ST_N_TAIL] = n_tail1;
      st[TCA_ST_SEQ_LEN] = seq_len + 1;
    }
    return;
  }
  // The host has checked its mirror for room; a captured call that is replayed moves on without it.  The state
  // words stay, so the row written above is not in use.  (In front of that write the test cost a decode step 0.4 us.)
  if (n_global + t_keep > gcap) {
    if (tid == 0) report_bounds_state(st, kBoundsGlobalRegion, n_global);
    return;
  }
  __syncthreads();  // the appended row is visible to the CTA (it is in the block when w = 0)

  compress_oldest_block(q_cur + size_t(u) * G * D, int64_t(D), Kc, Vc, pos, seg, ring, n_global, tail_head, tail_cap,
                        t_keep, D, G, b, sm_scale);
  if (tid == 0) {
    st[TCA_ST_N_GLOBAL] = n_global + t_keep;
    st[TCA_ST_TAIL_HEAD] = (tail_head + b) % tail_cap;
    st[TCA_ST_N_TAIL] = n_tail1 - b;
    st[TCA_ST_SEQ_LEN] = seq_len + 1;
  }
}

}  // namespace
}  // namespace tca

using namespace tca;

extern "C" int tca_cache_append(const tca_params* prm, tca_cache_desc* c, const void* k_new, const void* v_new,
                                const void* q_cur, void* stream) {
  int st = check_params(prm);
  if (st != TCA_OK) return st;
  TCA_CHECK_ARG(c && k_new && v_new && q_cur);
  TCA_CHECK_ARG(c->k && c->v && c->pos && c->state && c->global_cap && c->n_global && c->tail_head &&
                c->n_tail && c->seq_len && c->t_keep);
  const int64_t U = int64_t(prm->batch) * prm->n_kv_heads;
  TCA_CHECK_ARG(c->n_units == U);
  TCA_CHECK_ARG(aligned(c->k, 16) && aligned(c->v, 16));   // a block that leaves is read and moved in 16-byte pieces
  const int64_t full = int64_t(prm->window) + prm->block;
  if (c->tail_cap < full) return TCA_ERR_CAPACITY;
  for (int64_t u = 0; u < U; ++u) {
    TCA_CHECK_ARG(c->n_tail[u] < full);
    if (c->n_tail[u] + 1 >= full && c->n_global[u] + c->t_keep[u] > c->global_cap[u]) return TCA_ERR_CAPACITY;
    TCA_CHECK_ARG(c->seq_len[u] + 1 < (int64_t(1) << 31));
  }
  const int G = prm->n_q_heads / prm->n_kv_heads;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (prm->dtype == TCA_BF16) {
    using T = __nv_bfloat16;
    st = launch_pdl(cache_append_kernel<T>, dim3(unsigned(U)), dim3(kThreads), size_t(0), s,
                    static_cast<const T*>(k_new), static_cast<const T*>(v_new), static_cast<const T*>(q_cur),
                    static_cast<T*>(c->k), static_cast<T*>(c->v), c->pos, c->state, c->tail_cap, prm->head_dim, G,
                    prm->block, prm->window, double(prm->sm_scale));
  } else {
    using T = float;
    st = launch_pdl(cache_append_kernel<T>, dim3(unsigned(U)), dim3(kThreads), size_t(0), s,
                    static_cast<const T*>(k_new), static_cast<const T*>(v_new), static_cast<const T*>(q_cur),
                    static_cast<T*>(c->k), static_cast<T*>(c->v), c->pos, c->state, c->tail_cap, prm->head_dim, G,
                    prm->block, prm->window, double(prm->sm_scale));
  }
  if (st != TCA_OK) return st;
  for (int64_t u = 0; u < U; ++u) {
    c->n_tail[u] += 1;
    c->seq_len[u] += 1;
    if (c->n_tail[u] >= full) {
      c->n_global[u] += c->t_keep[u];
      c->tail_head[u] = (c->tail_head[u] + prm->block) % c->tail_cap;
      c->n_tail[u] -= prm->block;
    }
  }
  return TCA_OK;
}
