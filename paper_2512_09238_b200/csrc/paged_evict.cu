// tca_paged_evict: a unit keeps its sinks, its recent rows and, of the others, those that gathered the most attention
// weight; the kept rows behind the budget move into the holes in front of it.
//
// One cluster of CTAs per unit, each with a run of the unit's slots, four of which a thread reads at a time (a page holds a
// multiple of four).  The weights become order-preserving 32-bit keys, held in shared memory; the smallest kept key is
// found by radix selection, 8 or 11 bits at a time until nothing is left to tell, on histograms that the CTAs add to one
// another's shared memory.  The i-th hole below the budget takes the i-th kept row behind it: sources and destinations are disjoint, so rows move in any
// order, and no more of them than have to (keeping the order of slots would move all rows behind the first hole, through
// a staging buffer).  The pairs are put into shared memory by their number, equally many per CTA, so that the copies are
// dealt evenly wherever the rows lie.
// Bound by latency for short units, by memory for long ones: 8 bytes a row (weight, position) and twice a row's bytes for
// each that moves.  32 units of up to 1200 rows take 10 us (a CTA each); 32 of up to 64K rows cut to a third 48 us, 18 until the
// moves are known and 23 moving 119 MB (5.2 TB/s); one unit of 262144 rows, on its cluster's 16 SMs, 104.
#include <climits>

#include <cooperative_groups.h>

#include "paged_common.cuh"

namespace tca {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;          // more than 8 is not portable: evict_cluster() asks the device
constexpr int kMostSlots = 1 << 22;      // slots of a unit: one bit each has to fit a cluster's shared memory
constexpr int kHeld = 16 * 1024;         // slots of a CTA whose key and position are held; the others' are read again
constexpr int kPairs = 2 * 1024;         // moves of a CTA at a time
// Bits of a digit of the selection.  A CTA alone takes 11 (1200 rows: 12.4 against 13.7 us, the first two digits mostly
// tell); in a cluster every bin in use is sent to all, and 8 are better (units of up to
// 64K rows: 51.9 against 55.5 us).
constexpr int kBitsAlone = 11, kBitsCluster = 8, kBins = 1 << kBitsAlone, kSums = 1 << kBitsCluster;
constexpr uint32_t kSafe = 0xFFFFFFFFu;  // key of a sink or recent row; a NaN has the one below

struct EvictBuffers {
  uint4 *K, *V;
  int32_t* pos;
  float* mass;
  int shift;                             // log2 of a row's 16-byte pieces
};

__device__ __forceinline__ uint32_t mass_key(float x) {
  if (x != x) return kSafe - 1;
  const uint32_t u = __float_as_uint(x + 0.f);            // -0 becomes +0
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);      // at most that of +infinity, 0xFF800000
}

struct EvictShared {
  int max_pos[kMaxCluster], bad[kMaxCluster], safe[kMaxCluster];   // of every CTA of the cluster, written by each
  int2 counts[kMaxCluster];                                        // holes, kept rows behind the budget
  int scan[kWarps][2];
  alignas(16) unsigned hist[kBins];       // this CTA's
  alignas(16) unsigned sum[2][kSums];     // the cluster's, added up by all; two, so that one barrier per digit is enough
  unsigned picked;
  int need, equals;                       // left to find; keys equal to the threshold
  int equal[kMaxCluster];
};

// Dynamic shared memory: keys and positions [held_cap], moves (from, to) [pair_cap], a bit per slot: kept.
struct EvictSizes {
  int held_cap, pair_cap, words;
  int bytes() const { return held_cap * 8 + pair_cap * 8 + words * 4; }
};

__device__ __forceinline__ unsigned low_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

__global__ void __launch_bounds__(kThreads, 2)
evict_kernel(const __grid_constant__ EvictBuffers b, const __grid_constant__ PagedArgs args, int n_sink, int n_recent,
             const int32_t* __restrict__ budgets, EvictSizes sizes) {
  extern __shared__ __align__(16) uint32_t evict_smem[];
  __shared__ EvictShared sh;
  uint32_t* keys = evict_smem;
  int* held_pos = reinterpret_cast<int*>(evict_smem + sizes.held_cap);
  int2* pairs = reinterpret_cast<int2*>(evict_smem + 2 * sizes.held_cap);
  uint32_t* kept = evict_smem + 2 * sizes.held_cap + 2 * sizes.pair_cap;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = int(cluster.block_rank()), n_ctas = int(cluster.num_blocks());
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int u = int(blockIdx.x) / n_ctas;
  auto sync_all = [&] {                                   // a unit that is one CTA's needs no more than that CTA's barrier
    if (n_ctas > 1) cluster.sync(); else __syncthreads();
  };
  pdl_wait();
  pdl_launch_dependents();
  int4* st = args.state + u;
  const int len = paged_len(args, st->x), budget = budgets[u];
  if (len <= budget) return;                              // the whole cluster alike, before any barrier
  if (n_ctas > 1) cluster.barrier_arrive();
  const int per = ((len + n_ctas - 1) / n_ctas + 63) & ~63;   // a multiple of four slots, and of a word of bits
  const int s0 = min(len, rank * per), n = min(len, s0 + per) - s0, held = min((n + 3) & ~3, sizes.held_cap);

  // ---- one pass over positions and weights, four slots at a time
  int top = INT_MIN;
  bool bad = false;
#pragma unroll 4
  for (int i = tid * 4; i < n; i += kThreads * 4) {
    const int row = paged_row(args, u, s0 + i);
    if (row < 0) { bad = true; continue; }
    int4 pos = *reinterpret_cast<const int4*>(b.pos + row);
    const float4 w = *reinterpret_cast<const float4*>(b.mass + row);
    // (what lies behind the last row counts for nothing below)
    if (i + 1 >= n) pos.y = INT_MIN;
    if (i + 2 >= n) pos.z = INT_MIN;
    if (i + 3 >= n) pos.w = INT_MIN;
    top = max(max(top, max(pos.x, pos.y)), max(pos.z, pos.w));
    if (i < held) {
      *reinterpret_cast<uint4*>(keys + i) = make_uint4(mass_key(w.x), mass_key(w.y), mass_key(w.z), mass_key(w.w));
      *reinterpret_cast<int4*>(held_pos + i) = pos;
    }
  }
  top = __reduce_max_sync(0xffffffffu, top);
  bad = __any_sync(0xffffffffu, bad);
  if (lane == 0) { sh.scan[warp][0] = top; sh.scan[warp][1] = bad; }
  static_assert(kBins == 4 * kThreads, "four bins a thread");
  reinterpret_cast<uint4*>(sh.hist)[tid] = make_uint4(0, 0, 0, 0);
  static_assert(2 * kSums == kThreads, "a word a thread");
  sh.sum[tid / kSums][tid % kSums] = 0;
  __syncthreads();
  if (n_ctas > 1) cluster.barrier_wait();                 // every CTA of the cluster runs: its memory can be written
  if (tid < n_ctas) {
    int t = INT_MIN, any = 0;
    for (int w = 0; w < kWarps; ++w) { t = max(t, sh.scan[w][0]); any |= sh.scan[w][1]; }
    EvictShared* to = cluster.map_shared_rank(&sh, tid);
    to->max_pos[rank] = t;
    to->bad[rank] = any;
  }
  sync_all();
  int newest = INT_MIN, any_bad = 0;
  for (int c = 0; c < n_ctas; ++c) { newest = max(newest, sh.max_pos[c]); any_bad |= sh.bad[c]; }
  if (any_bad) {                                          // the whole cluster alike
    if (rank == 0 && tid == 0) report_paged(st, kPagedBadPage);
    return;
  }
  const int64_t recent_from = int64_t(newest) - n_recent; // positions above it are recent
  auto row_of = [&](int i) { return paged_row(args, u, s0 + i); };
  // Keys of slots s0 + i .. + 3 (i a multiple of four below n): a safe row has the highest.
  auto mark = [&](uint32_t key, int pos, int i) { return s0 + i < n_sink || pos > recent_from ? kSafe : key; };
  auto four = [&](int i) -> uint4 {
    if (i < held) return *reinterpret_cast<const uint4*>(keys + i);
    const int row = row_of(i);
    const int4 pos = *reinterpret_cast<const int4*>(b.pos + row);
    const float4 w = *reinterpret_cast<const float4*>(b.mass + row);
    return make_uint4(mark(mass_key(w.x), pos.x, i), mark(mass_key(w.y), pos.y, i + 1), mark(mass_key(w.z), pos.z, i + 2), mark(mass_key(w.w), pos.w, i + 3));
  };

  // ---- how many rows are safe?
  int safe = 0;
  for (int i = tid * 4; i < n; i += kThreads * 4) {
    uint4 k = four(i);
    if (i < held) {
      const int4 pos = *reinterpret_cast<const int4*>(held_pos + i);
      k = make_uint4(mark(k.x, pos.x, i), mark(k.y, pos.y, i + 1), mark(k.z, pos.z, i + 2), mark(k.w, pos.w, i + 3));
      *reinterpret_cast<uint4*>(keys + i) = k;
    }
    safe += (k.x == kSafe) + (i + 1 < n && k.y == kSafe) + (i + 2 < n && k.z == kSafe) + (i + 3 < n && k.w == kSafe);
  }
  safe = __reduce_add_sync(0xffffffffu, safe);
  if (lane == 0) sh.scan[warp][0] = safe;
  __syncthreads();
  if (tid < n_ctas) {
    int t = 0;
    for (int w = 0; w < kWarps; ++w) t += sh.scan[w][0];
    cluster.map_shared_rank(&sh, tid)->safe[rank] = t;
  }
  // ---- radix selection of the need-th largest key among the others
  uint32_t prefix = 0, least = kSafe;                     // least: the smallest key that is kept
  int need = 0;
  bool tie = false;                                       // not all keys equal to the least are kept
  const int most_bits = n_ctas > 1 ? kBitsCluster : kBitsAlone;
  for (int digit = 0, top = 32; top > 0; ++digit) {       // bits from `top` on are known
    const int bits = min(top, most_bits), shift = top - bits;
    const uint32_t mask = (1u << bits) - 1u;
    for (int i = tid * 4; i < n; i += kThreads * 4) {
      const uint4 k4 = four(i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t k = e == 0 ? k4.x : e == 1 ? k4.y : e == 2 ? k4.z : k4.w;
        const bool in = i + e < n && k != kSafe && (digit == 0 || (k >> top) == prefix);
        if (in) atomicAdd(&sh.hist[(k >> shift) & mask], 1u);   // (counting equal digits of a warp together first is slower)
      }
    }
    __syncthreads();
    const unsigned* counts = sh.hist;
    if (n_ctas > 1) {
      counts = sh.sum[digit & 1];
      if (tid < kSums) {
        // every CTA adds its counts to everybody's (read from the others after the barrier they took 1.2 us more a digit)
        const unsigned v = sh.hist[tid];
        if (v)
          for (int c = 0; c < n_ctas; ++c) atomicAdd(&cluster.map_shared_rank(&sh, c)->sum[digit & 1][tid], v);
      } else {
        sh.sum[(digit + 1) & 1][tid - kSums] = 0;         // read before the last barrier, added to after the next
      }
      cluster.sync();
    }
    if (digit == 0) {
      need = budget;
      for (int c = 0; c < n_ctas; ++c) need -= sh.safe[c];
      if (need < 0) {                                     // the whole cluster alike; nobody reads another's memory any more
        if (rank == 0 && tid == 0) report_paged(st, kPagedBudget);
        return;
      }
      if (need == 0) break;                               // none but the safe ones
    }
    // the bin at which the count from above reaches need, four bins per thread
    const int n_four = 1 << (most_bits - 2);              // (bins behind the last digit's are empty)
    const uint4 own = tid < n_four ? reinterpret_cast<const uint4*>(counts)[n_four - 1 - tid] : make_uint4(0, 0, 0, 0);
    const unsigned total = own.x + own.y + own.z + own.w;
    unsigned count = total;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const unsigned t = __shfl_up_sync(0xffffffffu, count, off);
      if (lane >= off) count += t;
    }
    if (lane == 31) sh.scan[warp][0] = int(count);
    __syncthreads();
    for (int w = 0; w < warp; ++w) count += unsigned(sh.scan[w][0]);
    int above = int(count - total);
    if (int(count) >= need && above < need) {
      int bin = (n_four - tid) * 4;
      unsigned in = 0;
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        if (above + int(in) >= need) break;
        above += int(in);
        in = i == 3 ? own.w : i == 2 ? own.z : i == 1 ? own.y : own.x;
        --bin;
      }
      sh.picked = bin;
      sh.need = need - above;
      sh.equals = int(in);
    }
    if (shift > 0) reinterpret_cast<uint4*>(sh.hist)[tid] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    prefix = (prefix << bits) | sh.picked;
    top = shift;
    need = sh.need;
    least = prefix << shift;
    tie = need != sh.equals;                              // the whole cluster alike
    if (!tie) break;                                      // the bin is kept whole
  }

  // ---- which slots are kept: keys from the least on, or of those equal to it the `need` lowest slots
  const int words = (n + 31) >> 5;
  int equals = 0;                                         // of the slots before: keys equal to the least
  if (tie) {
    if (tid < n_ctas) cluster.map_shared_rank(&sh, tid)->equal[rank] = int(sh.hist[sh.picked]);
    sync_all();
    for (int c = 0; c < rank; ++c) equals += sh.equal[c];
  }
  for (int i0 = 0; i0 < n; i0 += kThreads * 4) {
    const int i = i0 + tid * 4;
    const uint4 k4 = i < n ? four(i) : make_uint4(0, 0, 0, 0);
    unsigned nibble = 0, eq = 0;                          // of the four slots: kept, equal to the least
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t k = e == 0 ? k4.x : e == 1 ? k4.y : e == 2 ? k4.z : k4.w;
      if (i + e >= n) continue;
      if (k >= least) nibble |= 1u << e;
      if (k == least) eq |= 1u << e;
    }
    if (tie) {
      nibble &= ~eq;
      int incl = __popc(eq);
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += t;
      }
      __syncthreads();                                    // the counts of the chunk before have been read
      if (lane == 31) sh.scan[warp][0] = incl;
      __syncthreads();
      int mine = equals + incl - __popc(eq);
      for (int w = 0; w < kWarps; ++w) {
        if (w < warp) mine += sh.scan[w][0];
        equals += sh.scan[w][0];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if ((eq >> e) & 1u) nibble |= (mine++ < need ? 1u : 0u) << e;
    }
    unsigned word = nibble << (lane & 7) * 4;             // eight lanes make a word of 32 slots
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) word |= __shfl_xor_sync(0xffffffffu, word, off);
    if ((lane & 7) == 0 && (i >> 5) < words) kept[i >> 5] = word;
  }
  __syncthreads();
  // holes below the budget and kept rows behind it, of one word of 32 slots; each warp has a run of words
  auto holes_of = [&](int w) { return ~kept[w] & low_bits(n - w * 32) & low_bits(budget - s0 - w * 32); };
  auto late_of = [&](int w) { return kept[w] & ~low_bits(budget - s0 - w * 32); };
  const int w_begin = words * warp / kWarps, w_end = words * (warp + 1) / kWarps;
  int n_holes = 0, n_late = 0;
  for (int w = w_begin + lane; w < w_end; w += 32) {
    n_holes += __popc(holes_of(w));
    n_late += __popc(late_of(w));
  }
  n_holes = __reduce_add_sync(0xffffffffu, n_holes);
  n_late = __reduce_add_sync(0xffffffffu, n_late);
  if (lane == 0) { sh.scan[warp][0] = n_holes; sh.scan[warp][1] = n_late; }
  __syncthreads();
  if (tid < n_ctas) {
    int2 t = make_int2(0, 0);
    for (int w = 0; w < kWarps; ++w) { t.x += sh.scan[w][0]; t.y += sh.scan[w][1]; }
    cluster.map_shared_rank(&sh, tid)->counts[rank] = t;
  }
  sync_all();
  int hole0 = 0, late0 = 0, moves = 0;                    // numbers before this warp's words
  for (int w = 0; w < warp; ++w) { hole0 += sh.scan[w][0]; late0 += sh.scan[w][1]; }
  for (int c = 0; c < n_ctas; ++c) {
    if (c < rank) { hole0 += sh.counts[c].x; late0 += sh.counts[c].y; }
    moves += sh.counts[c].x;                              // as many kept rows lie behind the budget
  }
  // ---- the moves, dealt evenly by their number, in rounds if there are very many
  const int q = min(sizes.pair_cap, (moves + n_ctas - 1) / n_ctas);
  for (int first = 0; first < moves; first += q * n_ctas) {
    auto put = [&](int number, int i, bool to) {
      const int at = number - first;
      if (at < 0 || at >= q * n_ctas) return;
      int2* p = cluster.map_shared_rank(pairs, at / q) + at % q;
      (to ? p->y : p->x) = row_of(i);
    };
    int h = hole0, l = late0;
#pragma unroll 4
    for (int w = w_begin; w < w_end; ++w) {
      const unsigned hb = holes_of(w), lb = late_of(w);
      if ((hb >> lane) & 1u) put(h + __popc(hb & low_bits(lane)), w * 32 + lane, true);
      if ((lb >> lane) & 1u) put(l + __popc(lb & low_bits(lane)), w * 32 + lane, false);
      h += __popc(hb);
      l += __popc(lb);
    }
    sync_all();
    const int mine = min(q, moves - first - rank * q), pieces = mine > 0 ? mine << b.shift : 0;
    for (int p0 = tid; p0 < pieces; p0 += 4 * kThreads) {
      uint4 kv[4], vv[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = p0 + i * kThreads;
        if (p < pieces) {
          const int64_t at = (int64_t(pairs[p >> b.shift].x) << b.shift) + (p & ((1 << b.shift) - 1));
          kv[i] = b.K[at];
          vv[i] = b.V[at];
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = p0 + i * kThreads;
        if (p < pieces) {
          const int64_t at = (int64_t(pairs[p >> b.shift].y) << b.shift) + (p & ((1 << b.shift) - 1));
          b.K[at] = kv[i];
          b.V[at] = vv[i];
        }
      }
    }
    for (int p = tid; p < mine; p += kThreads) {
      const int2 m = pairs[p];
      b.pos[m.y] = b.pos[m.x];
      b.mass[m.y] = b.mass[m.x];
    }
    sync_all();
  }
  if (rank == 0 && tid == 0) st->x = budget;
}

}  // namespace
}  // namespace tca

using namespace tca;

namespace tca {
namespace {

// 16 if the current device can run clusters of 16 of the kernel with `bytes` of shared memory, else 8.  Asked once per device.
int evict_cluster(int bytes) {
  static std::atomic<uint64_t> wide{0}, narrow{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev >= 64) return 8;
  const uint64_t bit = uint64_t(1) << dev;
  if (wide.load(std::memory_order_relaxed) & bit) return 16;
  if (narrow.load(std::memory_order_relaxed) & bit) return 8;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(16);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = size_t(bytes);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 16;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  const bool can = cudaFuncSetAttribute(evict_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                   cudaOccupancyMaxActiveClusters(&n, evict_kernel, &cfg) == cudaSuccess && n > 0;
  cudaGetLastError();                    // a refusal is an answer here
  (can ? wide : narrow).fetch_or(bit, std::memory_order_relaxed);
  return can ? 16 : 8;
}

}  // namespace
}  // namespace tca

extern "C" int tca_paged_evict(const tca_params* prm, tca_paged_desc* c, int32_t n_sink, int32_t n_recent, const int32_t* budget,
                               void* stream) {
  const int st = check_paged(prm, c);
  if (st != TCA_OK) return st;
  TCA_CHECK_ARG(budget && aligned(budget, 4) && n_sink >= 0 && n_recent >= 0);
  const int64_t slots = int64_t(c->max_pages) * c->page_size;
  if (slots > kMostSlots) return TCA_ERR_UNSUPPORTED;
  // what the largest call can ask for: a bit for each of 512K slots beside the rest
  constexpr int kMostBytes = kHeld * 8 + kPairs * 8 + kMostSlots / 8 / 8;
  static_assert(kMostBytes + int(sizeof(EvictShared)) + 1024 <= 227 * 1024, "shared memory");
  if (allow_smem<evict_kernel>(kMostBytes) != TCA_OK) return TCA_ERR_CUDA;
  // CTAs per unit: as many as leave each two thousand slots, while the units do not fill the SMs with two each (and as many
  // as the bits of very long units need)
  const int most = slots > 2048 ? evict_cluster(kMostBytes) : 1;
  int n_ctas = 1;
  while (n_ctas < most && slots > int64_t(n_ctas) * 2048 &&
         (c->n_units * n_ctas <= 2 * sm_count() || slots > int64_t(n_ctas) * (kMostSlots / 8)))
    n_ctas *= 2;
  const int per = int(((slots + n_ctas - 1) / n_ctas + 63) & ~int64_t(63));
  EvictSizes sizes;
  sizes.held_cap = per < kHeld ? per : kHeld;
  sizes.pair_cap = per / 2 + 1 < kPairs ? per / 2 + 1 : kPairs;
  sizes.words = per / 32;
  EvictBuffers b;
  b.K = static_cast<uint4*>(c->k);
  b.V = static_cast<uint4*>(c->v);
  b.pos = c->pos;
  b.mass = c->mass;
  b.shift = 0;
  while ((16 << b.shift) < int64_t(prm->head_dim) * int64_t(elt_size(prm->dtype))) ++b.shift;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(c->n_units * n_ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = size_t(sizes.bytes());
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(n_ctas);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  TCA_CHECK_CUDA(cudaLaunchKernelEx(&cfg, evict_kernel, b, paged_args(c), int(n_sink), int(n_recent), budget, sizes));
  return TCA_OK;
}
