// Attention of up to two blocks of 128 query rows over a stream of 128-key tiles on the 5th-generation
// tensor cores (bf16 in, fp32 accumulators in TMEM, online softmax on the CUDA cores), shared by the packed
// prompt kernel and the drafted-tree kernel.  A Source says what the rows, tiles and masks are and
// what happens to a finished row.
//
// Two ways to use the two blocks:
//   kShared   both blocks attend to the same key tiles: 256 query rows per K/V tile brought in
//   !kShared  one block of query rows; the two "blocks" are two streams over alternate key tiles with a
//             softmax state each.  With 128 query rows or fewer there is no second block, and a single
//             stream would leave the tensor pipe idle during every softmax and the CUDA cores idle during
//             every product.
//
// 384 threads in three warpgroups: warp 0 TMA producer, warp 1 MMA issuer, warps 2 and 3 clean value tiles
// (below); warps 4-7 and 8-11 softmax of block 0 and 1, one thread per query row = TMEM lane.  The first
// warpgroup hands registers to the others (120 / 192 of 168 at launch), so that a thread holds its row
// of 128 scores.  TMEM: S0 | S1 | O0 | O1; the bf16 P of a tile overwrites the first half of its S and is
// the A operand of the second product.  Products are issued PV0 S0' PV1 S1' so that one block's softmax
// runs under the other's products; a stream step consumes one pair (V of this tile, K of the next of
// the same stream), which shares a full and an empty barrier.  P reaches the second product in two parts
// (96 keys, then 32).  O is rescaled only when a row maximum grew by more than 2^8 since the last time.
// Softmax statistics and O are fp32; P is rounded to bf16 because the product takes bf16 operands (half a
// step, 2^-8 of a weight), the row sum adds the unrounded weights.
//
// A masked weight is an exact zero, but zero times an infinity or NaN is not.  So before the second product
// of a tile that holds keys some row must not see, warps 2 and 3 clean its value tile in shared memory: rows
// nobody sees become zero, and a non-finite element of a row that some see and some do not becomes zero and
// is noted (Source::note); the epilogue adds it back to the rows that see it.  That costs nothing on the
// way: it runs under the tile's first product and softmax.
//
// Persistent: a CTA works through several items (a query tile against its keys), and the roles run ahead of
// one another across items.  While the softmax warps still write out an item, the next one's query tile and
// keys are on their way and its first scores are computed, so the latencies of starting an item are paid
// once per CTA.  The producer warp finds the items and hands them to the other roles through two slots.
//
// Every mbarrier wait is bounded; a wait that gives up raises the status word, lets copies land, frees
// TMEM and returns.
#pragma once
#include <cuda.h>

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "tensor_map.cuh"

namespace tca {

constexpr int kTcRows = 128, kTcKeys = 128;
constexpr int kTcThreads = 384;
constexpr int kTcRegsLean = 120, kTcRegsSoftmax = 192;
static_assert(128 * kTcRegsLean + 256 * kTcRegsSoftmax <= kTcThreads * 168, "more registers than the launch allocates");
constexpr int kTcHalfBytes = 128 * 128;        // 128 rows x 64 bf16: one swizzled box
constexpr float kTcRescale = 8.f;
constexpr int kTcPSplit = 6;                   // k-steps of 16 keys in the first part of P

// Writing rows held one per lane: four lanes exchange pieces of their rows, so that a store covers 64 or
// 128 contiguous bytes of each of 8 rows instead of 16 or 32 bytes of each of 32 (a store takes the memory
// pipe a cycle per row it touches).
struct TcRowOut {
  uint64_t row[4];       // the quad's rows; 0: not written
  __device__ __forceinline__ explicit TcRowOut(const void* mine) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      row[r] = __shfl_sync(0xffffffffu, static_cast<unsigned long long>(reinterpret_cast<uintptr_t>(mine)), (lane & ~3) + r);
  }
  // 4 x 4 transpose over the quad of kWords-word pieces: first with the lane two away, then with the
  // neighbour.  All of a step's exchanges are issued before the first result is used (one after the other
  // they cost their latency each, 40 clocks).  Afterwards piece r is row r's, number lane & 3 of it.
  template <int kWords>
  __device__ __forceinline__ void exchange(uint32_t* w) const {
    const int lane = threadIdx.x & 31;
    const bool up2 = lane & 2, up1 = lane & 1;
    uint32_t got[2 * kWords];
#pragma unroll
    for (int e = 0; e < 2 * kWords; ++e) got[e] = up2 ? w[e] : w[2 * kWords + e];
#pragma unroll
    for (int e = 0; e < 2 * kWords; ++e) got[e] = __shfl_xor_sync(0xffffffffu, got[e], 2);
#pragma unroll
    for (int e = 0; e < 2 * kWords; ++e) {
      w[e] = up2 ? got[e] : w[e];
      w[2 * kWords + e] = up2 ? w[2 * kWords + e] : got[e];
    }
#pragma unroll
    for (int e = 0; e < 2 * kWords; ++e) got[e] = up1 ? w[(e / kWords) * 2 * kWords + e % kWords] : w[(e / kWords) * 2 * kWords + kWords + e % kWords];
#pragma unroll
    for (int e = 0; e < 2 * kWords; ++e) got[e] = __shfl_xor_sync(0xffffffffu, got[e], 1);
#pragma unroll
    for (int e = 0; e < 2 * kWords; ++e) {
      uint32_t &lo = w[(e / kWords) * 2 * kWords + e % kWords], &hi = w[(e / kWords) * 2 * kWords + kWords + e % kWords];
      lo = up1 ? got[e] : lo;
      hi = up1 ? hi : got[e];
    }
  }
  // 128 bytes at byte offset `at` of every row (32-byte aligned); w: this lane's row's.  Whole warp.
  __device__ __forceinline__ void store32(uint32_t (&w)[32], int at) const {
    exchange<8>(w);
    at += (threadIdx.x & 3) * 32;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (row[r] == 0) continue;
      const uint32_t o[8] = {w[r * 8], w[r * 8 + 1], w[r * 8 + 2], w[r * 8 + 3], w[r * 8 + 4], w[r * 8 + 5], w[r * 8 + 6], w[r * 8 + 7]};
      ptx::st_global_32(reinterpret_cast<char*>(row[r]) + at, o);
    }
  }
  // 64 bytes at byte offset `at` of every row (16-byte aligned), from the first 16 words of w.
  __device__ __forceinline__ void store16(uint32_t (&w)[32], int at) const {
    exchange<4>(w);
    at += (threadIdx.x & 3) * 16;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (row[r] == 0) continue;
      *reinterpret_cast<uint4*>(reinterpret_cast<char*>(row[r]) + at) = make_uint4(w[r * 4], w[r * 4 + 1], w[r * 4 + 2], w[r * 4 + 3]);
    }
  }
};

template <int D>
struct TcLayout {
  static constexpr int NH = D / 64;
  static constexpr int kRing = D == 128 ? 5 : 9;          // K/V tiles in shared memory
  static constexpr int kPairs = kRing;                    // groups of loads (a V and a K tile) in flight, at least one tile each
  static constexpr int kTile = NH * kTcHalfBytes;         // a Q, K or V tile
  static constexpr int offQ = 0;
  static constexpr int offKV = 2 * kTile;
  static constexpr int offBar = offKV + kRing * kTile;
  static constexpr int kRaw = 8;                          // barriers of value tiles on their way to the cleaners; at most
  static_assert((kRing + 1) / 2 < kRaw, "value tiles in the ring");   // every other tile of the ring is a value tile, or all but one
  static constexpr int kBars = 6 + kRaw + 2 * kPairs + 2 + 4 + 2;
  static constexpr int bytes = offBar + 512 + 1024;       // barriers, alignment slack
  static_assert(bytes <= 227 * 1024 - 512, "shared memory");
  static_assert(kBars * 8 <= 512, "barrier block");
};

// Small shared state.  Item: what the producer warp hands to the other roles.
template <typename Item>
struct TcShared {
  uint32_t tmem;
  int abort;
  uint32_t dirty[2][2][4];   // per item slot: noted key rows of up to two tiles
  int any_dirty[2];
  int valid[2];
  Item item[2];
};

constexpr int kTcItemReaders = 1 + 2 + 8;   // issuer, cleaners, softmax warps

// Everything that needs no input: barriers and tensor memory.  Called by all threads before the dependency
// wait, so that it overlaps the end of the kernel before.
template <int D, typename Item>
__device__ __forceinline__ void flash_tc_setup(uint8_t* smem, TcShared<Item>* sh) {
  using L = TcLayout<D>;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::offBar);
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(bars + i, 1);                        // query tile full, empty
      ptx::mbar_init(bars + 2 + i, 1);                    // item full
      ptx::mbar_init(bars + 4 + i, kTcItemReaders);       // item empty
    }
    for (int i = 0; i < L::kRaw; ++i) ptx::mbar_init(bars + 6 + i, 1);
    uint64_t* full = bars + 6 + L::kRaw;
    for (int i = 0; i < L::kPairs; ++i) {
      ptx::mbar_init(full + i, 3);                        // K tile, V tile twice (the two cleaners, if it is cleaned)
      ptx::mbar_init(full + L::kPairs + i, 1);
    }
    uint64_t* s = full + 2 * L::kPairs;
    for (int h = 0; h < 2; ++h) {
      ptx::mbar_init(s + h, 1);
      ptx::mbar_init(s + 2 + 2 * h, 4);                   // one arrival per warp
      ptx::mbar_init(s + 3 + 2 * h, 4);
      ptx::mbar_init(s + 6 + h, 1);
    }
    ptx::fence_barrier_init();
    sh->abort = 0;
  }
  if (threadIdx.x < 32) {
    ptx::tmem_alloc(&sh->tmem, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
}

// Called by all 384 threads after flash_tc_setup and the dependency wait; returns with every thread after
// the last item.  Source:
//   struct Item                   plain data
//   void begin(lane)              whole warp, once: what find() needs
//   bool find(k, lane, item)      whole warp: the CTA's k-th item; false: there is none
//   void set(item)                all that follows is about this item
//   int  tiles(h)                 shared: tiles of block h; streams: all tiles (h ignored)
//   int  q_bytes(h)               bytes load_q(h) brings
//   void load_q(h, dst, bar)      issue the loads of block h's query tile
//   void load(t, is_v, dst, bar)  issue the loads of a K or V tile (kTile bytes)
//   void begin_row(row)           softmax threads, once: their row
//   int  row_key(h)               what last() needs of the row, worked out once per item
//   int  whole_tiles()            the first so many tiles are seen whole by every row
//   int  keys(h, t)               keys of tile t that some row of block h sees (1 .. 128)
//   int  last(key, t)             last key of tile t that the row sees (not asked for those)
//   int  clean(t)                 -1: nothing to clean; else rows of tile t that somebody sees
//   int  scan_from(t)             rows [scan_from(t), clean(t)) are searched for non-finite elements
//   int  note_slot(t)             which dirty[] entry a cleaned tile uses
//   void store(h, seen, m, l, dirty, read)  one finished row per thread, called by whole warps; seen:
//                                 the block had tiles; dirty: noted key rows or null; read(c, v): requests
//                                 columns 32 c .. of O (warp-wide; tc_wait_ld() before v is used)
template <int D, bool kShared, typename Source>
__device__ __forceinline__ void flash_tc(Source& src, uint8_t* smem, TcShared<typename Source::Item>* sh, float scale_log2e,
                                         int* status) {
  using L = TcLayout<D>;
  constexpr int kRing = L::kRing, kPairs = L::kPairs, kLead = kShared ? 1 : 2;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::offBar);
  uint64_t *bar_q = bars, *bar_q_empty = bars + 1, *bar_item = bars + 2, *bar_item_empty = bars + 4, *bar_raw = bars + 6;
  uint64_t *bar_full = bar_raw + L::kRaw, *bar_empty = bar_full + kPairs;
  uint64_t *bar_s = bar_empty + kPairs, *bar_p = bar_s + 2, *bar_pv = bar_p + 4;
  volatile int* abort_flag = &sh->abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t tmem_base = sh->tmem;
  // Loads of an item in ring order: the leading K tiles (1, or one per stream), then V_m and, if there is
  // one, K_m+lead for every tile m.  Groups: the leading tiles, then one per m.
  auto v_load = [&](int m, int nt) { const int lead = min(kLead, nt); return lead + m + min(m, nt - lead); };
  auto k_load = [&](int t, int nt) { return t < kLead ? t : v_load(t - kLead, nt) + 1; };
  auto warp_wait = [&](uint64_t* bar, uint32_t parity) -> bool {
    return __all_sync(0xffffffffu, ptx::mbar_wait(bar, parity, abort_flag));
  };
  // The k-th item as the other roles see it; false after the last one, or if a wait gave up.
  auto next_item = [&](int k) -> bool {
    if (!warp_wait(bar_item + (k & 1), uint32_t(k >> 1) & 1u)) return false;
    if (!sh->valid[k & 1]) return false;
    src.set(sh->item[k & 1]);
    return true;
  };
  auto item_done = [&](int k) {
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(bar_item_empty + (k & 1));
  };

  if (warp < 4) {
    ptx::reg_dealloc<kTcRegsLean>();
    if (warp == 0) {
      // ------------------------------------------------------------- producer: finds the items, brings the tiles
      int slot = 0;                   // ring slot of the next load
      int group = 0;                  // its group, counted over all items
      uint32_t cleaned = 0;           // value tiles handed to the cleaners
      int group_of[kRing];            // group of the tile a slot holds
#pragma unroll
      for (int i = 0; i < kRing; ++i) group_of[i] = -1;
      bool ok = true;
      auto wait_group = [&](int g) { return ptx::mbar_wait(bar_empty + g % kPairs, uint32_t(g / kPairs) & 1u, abort_flag); };
      // The status word is read here, behind the dependency wait: the kernel before may be what clears it.  Its trip
      // to memory is that of begin()'s loads.  If it stops the call there are no items.
      const int found_status = *reinterpret_cast<const volatile int*>(status);
      src.begin(lane);
      const bool stopped = __any_sync(0xffffffffu, stops_call(found_status));   // find() needs the whole warp
#pragma unroll 1
      for (int k = 0; ok; ++k) {
        typename Source::Item item;
        const bool have = !stopped && src.find(k, lane, item);
        if (k >= 2) ok = warp_wait(bar_item_empty + (k & 1), uint32_t((k >> 1) - 1) & 1u);
        if (!ok) break;
        if (lane == 0) {
          sh->valid[k & 1] = have ? 1 : 0;
          sh->item[k & 1] = item;
          for (int i = 0; i < 8; ++i) sh->dirty[k & 1][i >> 2][i & 3] = 0;
          sh->any_dirty[k & 1] = 0;
          ptx::mbar_arrive(bar_item + (k & 1));
        }
        if (!have) break;
        src.set(item);
        if (lane == 0) {
          const int n0 = src.tiles(0), n1 = kShared ? src.tiles(1) : 0, nt = kShared ? max(n0, n1) : n0;
          const bool two = kShared && n1 > 0;
          if (k > 0) ok = ptx::mbar_wait(bar_q_empty, uint32_t(k - 1) & 1u, abort_flag);
          if (ok) {
            ptx::mbar_arrive_expect_tx(bar_q, uint32_t(src.q_bytes(0) + (two ? src.q_bytes(1) : 0)));
            src.load_q(0, smem + L::offQ, bar_q);
            if (two) src.load_q(1, smem + L::offQ + L::kTile, bar_q);
          }
#pragma unroll 1
          for (int m = -1; m < nt && ok; ++m, ++group) {     // group m: V_m and K_m+lead; m = -1: the leading K tiles
            if (group >= kPairs) ok = wait_group(group - kPairs);
            uint64_t* full = bar_full + group % kPairs;
            const bool unclean = m >= 0 && src.clean(m) >= 0;
            if (!unclean) ptx::mbar_arrive(full);            // in the place of the second cleaner
#pragma unroll
            for (int j = 0; j < 2 && ok; ++j) {
              const bool is_v = m >= 0 && j == 0;
              const int t = m < 0 ? j : is_v ? m : m + kLead;
              if (t >= nt || (m < 0 && j >= kLead)) {        // no such tile: its arrival is still expected
                ptx::mbar_arrive(full);
                continue;
              }
              int held = -1;
#pragma unroll
              for (int i = 0; i < kRing; ++i)
                if (i == slot) { held = group_of[i]; group_of[i] = group; }
              if (held >= 0) ok = wait_group(held);          // the slot's previous tile must have been consumed
              if (!ok) break;
              uint64_t* bar = is_v && unclean ? bar_raw + cleaned++ % L::kRaw : full;
              ptx::mbar_arrive_expect_tx(bar, uint32_t(L::kTile));
              src.load(t, is_v, smem + L::offKV + slot * L::kTile, bar);
              slot = slot + 1 == kRing ? 0 : slot + 1;
            }
          }
        }
        ok = __all_sync(0xffffffffu, ok);
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------- MMA issuer (whole warp, one elected lane issues)
      constexpr uint32_t idesc_s = ptx::idesc_bf16(kTcRows, kTcKeys, false);
      constexpr uint32_t idesc_pv = ptx::idesc_bf16(kTcRows, D, true);
      const uint64_t dq = ptx::smem_desc_sw128(ptx::smem_u32(smem + L::offQ), 16, 1024);
      const uint64_t dk = ptx::smem_desc_sw128(ptx::smem_u32(smem + L::offKV), 16, 1024);             // K: K-major B
      const uint64_t dv = ptx::smem_desc_sw128(ptx::smem_u32(smem + L::offKV), kTcHalfBytes, 1024);   // V: MN-major B
      int base = 0, group = 0;               // first ring slot and group of the item
      uint32_t tile_count[2] = {0, 0};
      auto slot_of = [&](int n) { return (base + n) % kRing; };
      // Tiles that every row sees whole come first, and their steps are a loop of their own: the issuer's
      // instruction stream paces the products (with a run-time key count in one loop for all tiles a pair of
      // tiles took 4200 clocks instead of 3270).
      auto k_desc = [&](int n) { return dk + uint64_t(uint32_t(slot_of(n) * L::kTile) >> 4); };
      auto v_desc = [&](int n) { return dv + uint64_t(uint32_t(slot_of(n) * L::kTile) >> 4); };
      auto q_desc = [&](int h) { return dq + (kShared ? uint64_t(uint32_t(h * L::kTile) >> 4) : 0ull); };
      auto issue_s = [&](int h, int n) {
        const uint64_t a0 = q_desc(h), b0 = k_desc(n);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = (uint32_t(kk >> 2) * kTcHalfBytes + uint32_t(kk & 3) * 32u) >> 4;
          ptx::umma_ss_elect(tmem_base + h * 128u, a0 + off, b0 + off, idesc_s, kk > 0);
        }
      };
      auto issue_pv = [&](int h, int n, bool acc) -> bool {
        const uint64_t b0 = v_desc(n);
        const uint32_t parity = (h == 0 ? tile_count[0]++ : tile_count[1]++) & 1u;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          if (!warp_wait(bar_p + 2 * h + c, parity)) return false;
          ptx::tc_fence_after();
#pragma unroll
          for (int kk = (c == 0 ? 0 : kTcPSplit); kk < (c == 0 ? kTcPSplit : kTcKeys / 16); ++kk)
            ptx::umma_ts_elect(tmem_base + 256u + uint32_t(h * D), tmem_base + h * 128u + uint32_t(kk * 8),
                               b0 + uint32_t((kk * 2048) >> 4), idesc_pv, (acc || kk > 0) ? 1u : 0u);
        }
        return true;
      };
      // the same for any tile: only as many columns, and k-steps, in sixteens, as somebody sees
      auto issue_s_part = [&](int h, int n, int t) {
        const uint64_t a0 = q_desc(h), b0 = k_desc(n);
        const uint32_t idesc = ptx::idesc_bf16(kTcRows, 0, false) | (uint32_t((src.keys(h, t) + 15) >> 4 << 1) << 17);
#pragma unroll 1
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = (uint32_t(kk >> 2) * kTcHalfBytes + uint32_t(kk & 3) * 32u) >> 4;
          ptx::umma_ss_elect(tmem_base + h * 128u, a0 + off, b0 + off, idesc, kk > 0);
        }
      };
      auto issue_pv_part = [&](int h, int n, bool acc, int t) -> bool {
        const uint64_t b0 = v_desc(n);
        const uint32_t parity = (h == 0 ? tile_count[0]++ : tile_count[1]++) & 1u;
        const int steps = (src.keys(h, t) + 15) >> 4;
        if (!warp_wait(bar_p + 2 * h, parity) || !warp_wait(bar_p + 2 * h + 1, parity)) return false;
        ptx::tc_fence_after();
#pragma unroll 1
        for (int kk = 0; kk < steps; ++kk)
          ptx::umma_ts_elect(tmem_base + 256u + uint32_t(h * D), tmem_base + h * 128u + uint32_t(kk * 8),
                             b0 + uint32_t((kk * 2048) >> 4), idesc_pv, (acc || kk > 0) ? 1u : 0u);
        return true;
      };
#pragma unroll 1
      for (int k = 0; next_item(k); ++k) {
        const int n0 = src.tiles(0), n1 = kShared ? src.tiles(1) : 0, nt = kShared ? max(n0, n1) : n0;
        bool ok = warp_wait(bar_q, uint32_t(k) & 1u) && warp_wait(bar_full + group % kPairs, uint32_t(group / kPairs) & 1u);
        if (!ok) break;
        ptx::tc_fence_after();
#pragma unroll 1
        for (int h = 0; h < 2; ++h)
          if (kShared ? (h == 0 ? n0 : n1) > 0 : h < nt) {
            issue_s_part(h, kShared ? 0 : h, kShared ? 0 : h);
            ptx::umma_commit_elect(bar_s + h);
          }
        if (nt <= kLead) ptx::umma_commit_elect(bar_q_empty);      // that was the last use of the query tile
        ptx::umma_commit_elect(bar_empty + group % kPairs);
        ++group;
        int t = 0;
#pragma unroll 1
        for (const int fast = src.whole_tiles() - kLead; t < fast && ok; ++t, ++group) {
          ok = warp_wait(bar_full + group % kPairs, uint32_t(group / kPairs) & 1u);
          if (kShared) {
            for (int h = 0; h < 2 && ok; ++h) {
              if (h == 1 && n1 == 0) continue;
              ok = issue_pv(h, v_load(t, nt), t > 0);
              if (!ok) break;
              issue_s(h, k_load(t + 1, nt));
              ptx::umma_commit_elect(bar_s + h);                   // S ready implies PV done
            }
          } else {
            const int h = t & 1;
            if (ok) ok = issue_pv(h, v_load(t, nt), t > 1);
            if (!ok) break;
            issue_s(h, k_load(t + 2, nt));
            ptx::umma_commit_elect(bar_s + h);
          }
          if (!ok) break;
          if (t + 1 + kLead == nt) ptx::umma_commit_elect(bar_q_empty);      // the last scores have been issued
          ptx::umma_commit_elect(bar_empty + group % kPairs);
        }
#pragma unroll 1
        for (; t < nt && ok; ++t, ++group) {
          ok = warp_wait(bar_full + group % kPairs, uint32_t(group / kPairs) & 1u);
#pragma unroll 1
          for (int j = 0; j < (kShared ? 2 : 1) && ok; ++j) {
            const int h = kShared ? j : t & 1, mine = !kShared ? nt : h == 0 ? n0 : n1;   // tiles of this block / all
            if (t >= mine) continue;
            ok = issue_pv_part(h, v_load(t, nt), t >= kLead, t);
            if (!ok) break;
            const bool more = t + kLead < mine;
            if (more) issue_s_part(h, k_load(t + kLead, nt), t + kLead);
            ptx::umma_commit_elect(more ? bar_s + h : bar_pv + h);
          }
          if (!ok) break;
          if (t + 1 + kLead == nt) ptx::umma_commit_elect(bar_q_empty);
          ptx::umma_commit_elect(bar_empty + group % kPairs);
        }
        if (!ok) break;
        base = slot_of(2 * nt);
        item_done(k);
      }
    } else {
      // ------------------------------------------------------------- cleaning of value tiles (warps 2 and 3: 64 rows each)
      // Such a tile arrives on a barrier of its own and joins its group when both warps are done with it.
      uint32_t cleaned = 0;
      int base = 0, group = 0;
#pragma unroll 1
      for (int k = 0; next_item(k); ++k) {
        const int n0 = src.tiles(0), n1 = kShared ? src.tiles(1) : 0, nt = kShared ? max(n0, n1) : n0;
        bool ok = true;
        for (int t = 0; t < nt && ok; ++t) {
          const int seen = src.clean(t);
          if (seen < 0) continue;
          ok = warp_wait(bar_raw + cleaned % L::kRaw, (cleaned / L::kRaw) & 1u);
          if (!ok) break;
          ++cleaned;
          uint8_t* tile = smem + L::offKV + (base + v_load(t, nt)) % kRing * L::kTile;
          // One 16-byte piece per lane; the swizzle only permutes the pieces within a row.  The search takes
          // the maximum of |x| over all pieces of the lane (NaN wins over everything): 2 instructions per
          // 4 bytes, and only if that is not finite the pieces are looked at one by one.
          constexpr int kPieces = L::NH * 8;                 // per row
          auto piece = [&](int i) {                          // i-th piece of the rows this warp takes, rows alternate between the two
            const int r = 2 * (i / kPieces) + (warp - 2), c = i % kPieces;
            return reinterpret_cast<uint4*>(tile + (c >> 3) * kTcHalfBytes + r * 128 + (c & 7) * 16);
          };
          const int z0 = (max(seen, 0) + 1 - (warp - 2)) / 2;      // first of this warp's rows that nobody sees
          const int s0 = (src.scan_from(t) + 1 - (warp - 2)) / 2;  // first of its rows to search
          __nv_bfloat162 top = __floats2bfloat162_rn(0.f, 0.f);
          for (int i0 = s0 * kPieces + lane; i0 < z0 * kPieces; i0 += 32 * 8) {
            uint4 v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = i0 + 32 * j < z0 * kPieces ? *piece(i0 + 32 * j) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const uint32_t* w = &v[j].x;
#pragma unroll
              for (int e = 0; e < 4; ++e) top = __hmax2_nan(top, __habs2(reinterpret_cast<const __nv_bfloat162&>(w[e])));
            }
          }
          const uint32_t tw = reinterpret_cast<const uint32_t&>(top);
          if ((tw & 0x7f80u) == 0x7f80u || (tw & 0x7f800000u) == 0x7f800000u) {
            for (int i = s0 * kPieces + lane; i < z0 * kPieces; i += 32) {
              uint4 v = *piece(i);
              uint32_t* w = &v.x;
              bool hit = false;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((w[e] & 0x7f80u) == 0x7f80u) { w[e] &= 0xffff0000u; hit = true; }
                if ((w[e] & 0x7f800000u) == 0x7f800000u) { w[e] &= 0xffffu; hit = true; }
              }
              if (!hit) continue;
              *piece(i) = v;
              const int r = 2 * (i / kPieces) + (warp - 2);
              atomicOr(&sh->dirty[k & 1][src.note_slot(t)][r >> 5], 1u << (r & 31));
              sh->any_dirty[k & 1] = 1;
            }
          }
          const int z1 = (((seen + 15) & ~15) + 1 - (warp - 2)) / 2;   // the product reads whole k-steps
          for (int i = z0 * kPieces + lane; i < z1 * kPieces; i += 32) *piece(i) = make_uint4(0, 0, 0, 0);
          ptx::fence_proxy_async_smem();                     // the product reads the tile through the async proxy
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar_full + (group + 1 + t) % kPairs);
        }
        if (!ok) break;
        base = (base + 2 * nt) % kRing;
        group += nt + 1;
        item_done(k);
      }
    }
  } else {
    ptx::reg_alloc<kTcRegsSoftmax>();
    // ------------------------------------------------------------- softmax, one row per thread
    const int h = (warp - 4) >> 2;
    const int quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t lane_addr = tmem_base + (uint32_t(quarter * 32) << 16);
    const uint32_t s_addr = lane_addr + h * 128u, o_addr = lane_addr + 256u + uint32_t(h * D);
    const uint64_t scale2 = ptx::pack2(scale_log2e, scale_log2e);
    uint32_t tile_count = 0, item_count = 0;
    src.begin_row(row);
    for (int k = 0; !*abort_flag && next_item(k); ++k) {
      const int nt = src.tiles(kShared ? h : 0);
      const int mine = kShared ? nt : (nt - h + 1) / 2;      // tiles of this block / stream
      const int row_key = src.row_key(h);
      float m_run = -INFINITY, m_used = -INFINITY, l = 0.f;
      bool ok = true;
      // lazy rescale of the accumulator to a maximum that grew by more than 2^8.  TMEM access is warp-wide, so
      // the warp votes; but a row whose own maximum did not grow that far keeps its scale (times one is exact):
      // otherwise its rounding would follow its neighbours' scores, and those may be another sequence's or
      // rows of the tile that hold no query at all
      auto rescale = [&](float mx, bool started) {
        m_run = fmaxf(m_run, mx * scale_log2e);
        const bool grew = m_run > m_used + kTcRescale;
        if (__any_sync(0xffffffffu, grew)) {
          const float alpha = !grew ? 1.f : m_used == -INFINITY ? 0.f : ptx::fast_exp2(m_used - m_run);
          if (started) {
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
              uint32_t o[32];
              ptx::tmem_ld32(o_addr + c * 32, o);
              ptx::tc_wait_ld();
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
              ptx::tmem_st32(o_addr + c * 32, o);
            }
            ptx::tc_wait_st();
          }
          l *= alpha;
          if (grew) m_used = m_run;
        }
      };
      auto announce = [&](int part) {
        ptx::tc_wait_st();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar_p + 2 * h + part);
      };
      const int whole = kShared ? min(src.whole_tiles(), mine) : (src.whole_tiles() - h + 1) / 2;   // they come first
      int it = 0;
#pragma unroll 1
      for (; it < whole; ++it) {
        ok = warp_wait(bar_s + h, tile_count++ & 1u);
        if (!ok) break;
        ptx::tc_fence_after();
        uint32_t v[kTcKeys];
#pragma unroll
        for (int c = 0; c < kTcKeys / 32; ++c)
          ptx::tmem_ld32(s_addr + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&v[c * 32]));
        ptx::tc_wait_ld();
        float mx;
        {
          float mx8[8];
#pragma unroll
          for (int a = 0; a < 8; ++a) mx8[a] = fmaxf(__uint_as_float(v[2 * a]), __uint_as_float(v[2 * a + 1]));
#pragma unroll
          for (int k = 16; k < kTcKeys; k += 16)
#pragma unroll
            for (int a = 0; a < 8; ++a)
              mx8[a] = ptx::max3(mx8[a], __uint_as_float(v[k + 2 * a]), __uint_as_float(v[k + 2 * a + 1]));
          mx = fmaxf(fmaxf(ptx::max3(mx8[0], mx8[1], mx8[2]), ptx::max3(mx8[3], mx8[4], mx8[5])), fmaxf(mx8[6], mx8[7]));
        }
        rescale(mx, it > 0);
        const float neg_m = (m_used == -INFINITY) ? 0.f : -m_used;
        const uint64_t neg_m2 = ptx::pack2(neg_m, neg_m);
        uint64_t sum2[2] = {0ull, 0ull};
        // eight groups of 16 scores; a group's store is issued only after the next group's arithmetic, so it
        // never waits for exponentials still in flight
#pragma unroll
        for (int g = 0; g < 8; ++g) {
#pragma unroll
          for (int jj = 0; jj < 8; ++jj) {
            const int j = g * 8 + jj;
            float xl, xh;
            ptx::unpack2(ptx::fma2(ptx::pack2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), scale2, neg_m2), xl, xh);
            const float el = ptx::fast_exp2(xl), eh = ptx::fast_exp2(xh);
            sum2[j & 1] = ptx::add2(sum2[j & 1], ptx::pack2(el, eh));
            v[j] = ptx::pack_bf16x2(el, eh);   // entry j is never read again (j <= 2j)
          }
          if (g == kTcPSplit + 1) {            // the first part was stored at least one group ago
            announce(0);
          }
          if (g >= 1) ptx::tmem_st8(s_addr + (g - 1) * 8, &v[(g - 1) * 8]);
        }
        ptx::tmem_st8(s_addr + 56, &v[56]);
        announce(1);
        float s0, s1, s2, s3;
        ptx::unpack2(sum2[0], s0, s1);
        ptx::unpack2(sum2[1], s2, s3);
        l += (s0 + s1) + (s2 + s3);
      }
#pragma unroll 1
      for (; it < mine && ok; ++it) {
        const int t = kShared ? it : 2 * it + h;
        ok = warp_wait(bar_s + h, tile_count++ & 1u);
        if (!ok) break;
        ptx::tc_fence_after();
        // A tile that some row does not see all of (the diagonal, the end of a run): the 32-key groups that
        // somebody sees, in a compact loop that reads the scores twice.
        const int hi = src.last(row_key, t), groups = (src.keys(h, t) + 31) >> 5;
        float mx = -INFINITY;
#pragma unroll 1
        for (int c = 0; c < groups; ++c) {
          uint32_t v[32];
          ptx::tmem_ld32(s_addr + c * 32, v);
          ptx::tc_wait_ld();
          const int last = hi - c * 32;
#pragma unroll
          for (int k = 0; k < 32; ++k)
            if (k <= last) mx = fmaxf(mx, __uint_as_float(v[k]));
        }
        rescale(mx, it > 0);
        const float neg_m = (m_used == -INFINITY) ? 0.f : -m_used;
        float sum = 0.f;
#pragma unroll 1
        for (int c = 0; c < groups; ++c) {
          uint32_t v[32];
          ptx::tmem_ld32(s_addr + c * 32, v);
          ptx::tc_wait_ld();
          const int last = hi - c * 32;
#pragma unroll
          for (int k = 0; k < 32; k += 2) {    // a key the row does not see has weight 0, whatever its score
            const float el = k <= last ? ptx::fast_exp2(fmaf(__uint_as_float(v[k]), scale_log2e, neg_m)) : 0.f;
            const float eh = k + 1 <= last ? ptx::fast_exp2(fmaf(__uint_as_float(v[k + 1]), scale_log2e, neg_m)) : 0.f;
            sum += el + eh;
            v[k / 2] = ptx::pack_bf16x2(el, eh);
          }
          ptx::tmem_st16(s_addr + c * 16, v);  // over scores that have been read
        }
        announce(0);
        announce(1);
        l += sum;
      }
      if (ok && mine > 0) ok = warp_wait(bar_pv + h, item_count++ & 1u);   // committed after the last PV
      if (!ok) break;
      ptx::tc_fence_after();
      src.store(h, mine > 0, m_used, l, sh->any_dirty[k & 1] ? &sh->dirty[k & 1][0][0] : nullptr,
                [&](int c, uint32_t (&v)[32]) { ptx::tmem_ld32(o_addr + c * 32, v); });
      ptx::tc_fence_before();       // the reads of O precede the next item's products (through the P barriers)
      item_done(k);
    }
  }
  // ------------------------------------------------------------- teardown
  ptx::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // a wait that gave up outranks a failed range check: there is no result
    if (kDebugBounds && tid == 0) atomicCAS(status, kStatusBounds, kStatusTimeout);
    ptx::abort_teardown(status, tid);      // status word, then time for copies in flight to land
  }
  if (warp == 0) ptx::tmem_dealloc(tmem_base, 512);
}

}  // namespace tca
