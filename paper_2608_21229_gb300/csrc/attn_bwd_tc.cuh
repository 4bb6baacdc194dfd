// attn_bwd_tc.cuh -- the gradients of the joint attention (attn_bwd.cuh) on
// tcgen05 MMAs over CTA pairs (cta_group::2, M = 256), head dim 128 or 64.
//
// attn_bwd_keys_kernel: 256 keys of one head, 128 per CTA; query tiles of 128 rows:
//   S^T = K Q^T, dP^T = V dO^T          A = the keys' rows (kept), B = the tile's rows
//   P^T = exp2(S^T scale log2 e - lse log2 e), dS^T = P^T (dP^T - delta)
//   dV += P^T dO, dK += dS^T Q          A = P^T, dS^T in tensor memory, B = the tile's rows
// attn_bwd_queries_kernel: 256 queries of one head; key tiles of 128 rows:
//   S = Q K^T, dP = dO V^T, dS = P (dP - delta), dQ += dS K
//
// The B operand of a pair's MMA is split along N between its CTAs, so a tile is
// held twice: rows [64 r, 64 r + 64) of it in CTA r for the products over the
// head dim, columns [D/2 r, D/2 (r + 1)) of all 128 rows for the products
// over the rows.  Per tile of 128 queries and 256 keys (512 tensor cycles a
// product at D = 128) each CTA's tensor core then reads 128 KB of its shared memory in the
// keys kernel's 2048 cycles, and 64 KB arrive: three quarters of the 128 bytes a cycle that
// the memory gives.  One CTA alone (M = 128) would need 320 KB in that time.
//
// Tensor memory (512 columns), keys kernel: S^T [0, 128), dP^T [128, 256), dV
// [256, 384), dK [384, 512); P^T and dS^T as bf16 over the scores they come from.
// The tensor core's order of work is
//   S_0 dP_0 | dV_0 S_1 | dK_0 dP_1 | dV_1 S_2 | dK_1 dP_2 | ...
// so that P_i is found from S_i while dK_i-1 and dP_i run, and dS_i from dP_i while
// dV_i and S_i+1 run: each has 1024 tensor cycles, with one buffer each.  At head dim 64
// these are 512, less than the way from S to P to the next S takes, and there is room
// for two S: S_i+2 follows dV_i.
// Queries kernel: S [0, 128), dP twice [128, 384), dQ [384, 512); P never leaves
// the registers, S is free as soon as it is read, and the order is
//   S_i dP_i dQ_i-1 | S_i+1 dP_i+1 dQ_i | ...
// across items: an item's first S and dP are issued inside the item before it.
//
// Warps: 0-7 scores (warp w: lanes 32 (w % 4).., columns 64 (w / 4)..; P and dS are
// written over the columns that the same warp has read), 8 TMA producer, 9 MMAs
// (leader), 10 statistics of the query tiles (keys kernel), 11 items.
//
// The queries kernel is launched first and the keys kernel as its programmatic
// dependent: the keys kernel's CTAs take SMs as the queries kernel's leave, which they
// need not wait for, only before their own end.  What both read (inputs, statistics,
// counters) was there when the queries kernel passed its wait, which it says with a
// ticket that the keys kernel's CTAs acquire (kBwdPassed).  Items are handed out to
// whichever pair is free.
//
// What bounds them: at D = 128 the tensor pipe (with many tiles an item, under the power
// cap), at D = 64 the score warps and as long a chain from one S to the next (arrivals,
// MMAs, commits).  Measured, each alone on the GPU and after a pause, at a clock that the
// power cap does not hold for long:
//                                    keys kernel              queries kernel
//   cycles per tile, D = 128         2250 (MMAs: 2048)        1690 (1536)
//   cycles per tile, D = 64          1710 (1024)              1510 (768)
//   and between items                5700 (its output)        2500
//   24 heads of 128, 1280 queries    78 us, 1345 TFLOP/s      58 us, 1355 TFLOP/s
//     and 3328 keys                  of its four products     of its three
//   4608 queries, 25088 keys         1403 us, 2025            1067 us, 2000
//   16 heads of 64, three requests   280 us, 1290             240 us, 1130
//     of 9431 rows together
// One after the other with the pass over the outputs, call after call: 128, 2820 and 531 us, at
// 1910, 1575 and 1995 MHz (sampled).  Of the 4.44 M cycles that 2820 us are, the seven
// products' MMAs take 3.99 M.
//
// All waits are bounded as in attn_tc2_kernel, and the teardown is that kernel's:
// loads complete on the leader's barriers, which it arms for both CTAs' bytes.
#pragma once
#include "attn_bwd.cuh"
#include "attn_tc.cuh"

namespace rc {

struct BwdMaps {
  // 64 rows x 64 columns (128-byte swizzle) of q, dO, ka, va, kb, vb; 128 rows x
  // D / 2 columns of two of them (keys kernel: dO, q; queries kernel: ka, kb)
  CUtensorMap q, d_o, ka, va, kb, vb, cols0, cols1;
};

namespace bwd {
using tc::Ctl;
constexpr int kThreads = 32 * 12;
constexpr int kScoreWarps = 8, kProducerWarp = 8, kMmaWarp = 9, kStatWarp = 10, kItemWarp = 11;
constexpr int kTile = 128;   // rows of a tile
constexpr int kBlock = 256;  // rows of an item
constexpr int kStatSlots = 2;
constexpr int kItemSlots = 2;

// What a CTA keeps of an item is its 128 rows of two operands: X (K or Q), of S, and
// Y (V or dO), of dP.  R: a tile's rows, half of them in each CTA, of S and of dP;
// C: its columns.
//   keys kernel     X and Y once, loaded together; R of S and dP together; an area where
//                   dK and dV are staged on their way out
//   queries kernel  X and Y twice, so that an item's first S and dP are issued inside
//                   the item before it, whose X then takes its dQ on its way out
// At head dim 64 a tile is half as many bytes and takes less time, so its rings are
// deeper (a load takes about as long as a tile).  At 128 the queries kernel's R are loads
// of their own, so that each has all the time between its uses; at 64 they are one, for
// the MMA warp, whose waits and commits take the longer the shorter a tile is.
template <int D, bool kKeys>
struct Smem {
  static constexpr uint32_t kOwn = 128 * D * 2;  // this CTA's 128 rows of one operand
  static constexpr uint32_t kHalf = 64 * D * 2;  // half a tile's rows, or half its columns
  static constexpr int kXSlots = kKeys ? 1 : 2, kYSlots = kXSlots;
  static constexpr uint32_t kXSlot = kKeys ? kOwn : 32768;  // (32 rows x 64 columns a warp are staged in it)
  static constexpr uint32_t kXBytes = kKeys ? 2 * kOwn : kOwn;  // one CTA's bytes of a load: with Y in the keys kernel
  static constexpr int kSBufs = kKeys && D == 64 ? 2 : 1;       // S in tensor memory
  static constexpr int kSlots = D == 64 ? 4 : 2;                // of each ring of a tile
  static constexpr bool kRApart = !kKeys && D == 128;           // R of S and of dP are loads of their own
  static constexpr uint32_t kR1Bytes = kRApart ? kHalf : 2 * kHalf;
  static constexpr uint32_t kCBytes = (kKeys ? 2 : 1) * kHalf;
  static constexpr uint32_t kX = 0, kY = kX + kXSlots * kXSlot, kR1 = kY + kYSlots * kOwn, kR2 = kR1 + kSlots * kR1Bytes,
                            kC = kR2 + (kRApart ? kSlots * kHalf : 0), kStage = kC + kSlots * kCBytes,
                            kStat = kStage + (kKeys ? kScoreWarps * 4096 : 0);
  static constexpr uint32_t kBars = kStat + (kKeys ? kStatSlots * 1024 : 0);
  // barriers; those of loads first: X, Y, rows of S, rows of dP, columns (Y and rows of dP: where they are loads of their own)
  static constexpr int kYLoads = kKeys ? 0 : kYSlots, kR2Loads = kRApart ? kSlots : 0;
  static constexpr int kPBufs = kKeys ? 1 : 2, kHalves = kKeys && kSBufs == 1 ? 1 : 0, kStats = kKeys ? kStatSlots : 0;
  static constexpr int kXFull = 0, kYFull = kXFull + kXSlots, kR1Full = kYFull + kYLoads, kR2Full = kR1Full + kSlots,
                       kCFull = kR2Full + kR2Loads, kXEmpty = kCFull + kSlots, kYEmpty = kXEmpty + kXSlots, kR1Empty = kYEmpty + kYLoads,
                       kR2Empty = kR1Empty + kSlots, kCEmpty = kR2Empty + kR2Loads, kSDone = kCEmpty + kSlots, kPDone = kSDone + kSBufs,
                       kSHalf = kPDone + kPBufs, kSUsed = kSHalf + kHalves, kDsFull = kSUsed + kSBufs, kAccFree = kDsFull + kPBufs,
                       kAccDone = kAccFree + 1, kStatFull = kAccDone + 1, kStatEmpty = kStatFull + kStats, kItemFull = kStatEmpty + kStats,
                       kItemEmpty = kItemFull + kItemSlots, kItemIn = kItemEmpty + kItemSlots, kItemPeer = kItemIn + kItemSlots,
                       kMmaDone = kItemPeer + kItemSlots, kNumBars = kMmaDone + 1;
  // warps that read each item from a CTA's ring: its producer, score (and statistics)
  // warps, and the leader's MMA warp
  static constexpr int kItemTakers = 1 + kScoreWarps + (kKeys ? 1 : 0);
  static constexpr uint32_t kTmemHolder = kBars + 8 * kNumBars;
  static constexpr uint32_t kAbort = kTmemHolder + 4, kPeerAbort = kAbort + 4;
  static constexpr uint32_t kLoadRec = kPeerAbort + 4;  // each CTA's loads: X, Y, rows of S, rows of dP, columns
  static constexpr uint32_t kItemRing = (kLoadRec + 40 + 15u) & ~15u;
  static constexpr uint32_t kUsed = kItemRing + 48 * kItemSlots;
  static constexpr uint32_t kMaxDynamic = 232448;
  static constexpr uint32_t kDynamic = kUsed + 1024 < kMaxDynamic ? kUsed + 1024 : kMaxDynamic;
  static_assert(kUsed <= kMaxDynamic, "shared-memory layout too large");
};

// The MMAs of one product; a descriptor counts in units of 16 bytes.  Products over the
// head dim: A is this CTA's 128 rows, B 64 rows of the tile, both in boxes of 64 columns.
template <int D>
__device__ __forceinline__ void mma_rows(uint32_t d_tmem, uint64_t a, uint64_t b) {
  constexpr uint32_t kIdesc = idesc_bf16_f32(256, kTile, false);
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk)
    tc2_mma_ss(d_tmem, a + (((kk >> 2) * 16384u + (kk & 3) * 32u) >> 4), b + (((kk >> 2) * 8192u + (kk & 3) * 32u) >> 4), kIdesc,
               kk > 0 ? 1u : 0u);
}
// Products over a tile's rows: A is P or dS (128 weights a row, bf16 in tensor memory, the
// second 64 at +64 columns), B the tile's columns.  Part 0, 1: the first or second 32 of each 64 weights; -1: all.
template <int D, int kPart>
__device__ __forceinline__ void mma_cols(uint32_t d_tmem, uint32_t w_tmem, uint64_t b, uint32_t accumulate) {
  constexpr uint32_t kIdesc = idesc_bf16_f32(256, D, true);
#pragma unroll
  for (int kk = 0; kk < kTile / 16; ++kk)
    if (kPart < 0 || ((kk >> 1) & 1) == kPart)
      tc2_mma_ts(d_tmem, w_tmem + static_cast<uint32_t>((kk >> 2) * 64 + (kk & 3) * 8), b + ((16u * D * kk) >> 4), kIdesc,
                 kk > 0 ? 1u : accumulate);
}
template <int D>
__device__ __forceinline__ uint64_t cols_desc(uint32_t addr) {
  return D == 64 ? sdesc_sw64(addr, 128 * D, 512) : sdesc_sw128(addr, 128 * D, 1024);
}

// 64 columns of this thread's lane.
__device__ __forceinline__ void load64(uint32_t t, float (&s)[64]) {
  uint32_t r0[32], r1[32];
  tmem_ld32(t, r0);
  tmem_ld32(t + 32, r1);
  tmem_wait_ld(r0);
  tmem_wait_ld(r1);
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    s[i] = __uint_as_float(r0[i]);
    s[32 + i] = __uint_as_float(r1[i]);
  }
}

// One warp's 32 rows x 64 columns of bf16, or 32 of fp32 (eight chunks of 16 bytes of each
// row), through shared memory, so that whole 128-byte lines are written.
struct RowsOut {
  uint32_t stage;  // this warp's 4 KB
  int lane;
  __device__ __forceinline__ void put(int chunk, uint4 v) const {
    st_shared_v4(stage + 128u * lane + (static_cast<uint32_t>(chunk ^ (lane & 7)) << 4), v);
  }
  __device__ __forceinline__ uint4 get(int chunk) const {
    return ld_shared_v4(stage + 128u * lane + (static_cast<uint32_t>(chunk ^ (lane & 7)) << 4));
  }
  // rows [from, rows) of the warp come from src + row * stride, zeros elsewhere
  template <typename T>
  __device__ __forceinline__ void fetch(const T* src, int64_t stride, int from, int rows) const {
    const int r0 = lane >> 3, ch = lane & 7;
    uint4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = 4 * i + r0;
      v[i] = r >= from && r < rows ? *reinterpret_cast<const uint4*>(src + r * stride + 16 / sizeof(T) * ch) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = 4 * i + r0;
      st_shared_v4(stage + 128u * r + (static_cast<uint32_t>(ch ^ (r & 7)) << 4), v[i]);
    }
    __syncwarp();
  }
  // rows [0, rows) of the warp go to dst + row * stride
  template <typename T>
  __device__ __forceinline__ void flush(T* dst, int64_t stride, int rows) const {
    __syncwarp();
    const int r0 = lane >> 3, ch = lane & 7;
#pragma unroll 4
    for (int i = 0; i < 8; ++i) {
      const int r = 4 * i + r0;
      const uint4 v = ld_shared_v4(stage + 128u * r + (static_cast<uint32_t>(ch ^ (r & 7)) << 4));
      if (r < rows) *reinterpret_cast<uint4*>(dst + r * stride + 16 / sizeof(T) * ch) = v;
    }
    __syncwarp();
  }
};

// An item: rows [row0, row0 + rows) of one head and nt tiles of the other side.
struct Item {
  int head, row0, rows, nt;
  int v[5];  // keys kernel: first query row, query rows, in_b, add_from, add_row0; queries kernel: a_row0, a_len, b_row0, b_len, tiles of A
};

// What both kernels set up before their roles part.
template <typename L>
struct Cta {
  uint32_t base, rank;
  uint8_t* ptr;
  int warp, lane;
  bool leader;
  Ctl ctl;
  uint32_t tmem;
  __device__ __forceinline__ uint32_t bar(int i) const { return base + L::kBars + 8u * static_cast<uint32_t>(i); }
  __device__ __forceinline__ uint32_t lbar(int i) const { return mapa_shared(bar(i), 0); }
  __device__ __forceinline__ bool wait(int i, int n, int where) const {  // completion n (0, 1, ..) of barrier i
    return tc::wait_one(bar(i), static_cast<uint32_t>(n) & 1u, ctl, where);
  }
  __device__ __forceinline__ bool wait_all(int i, int n, int where) const { return __all_sync(0xffffffffu, wait(i, n, where)); }
  __device__ __forceinline__ bool done(int i, int n) const { return mbar_test_wait(bar(i), static_cast<uint32_t>(n) & 1u); }
  // Items reach the warps through a ring in the shared memory of both CTAs, decoded:
  // the leader's item warp (one lane) writes item k to both, the follower's tells its CTA
  // that it has come, and the leader when its CTA is done with it.  All other warps meet
  // at barriers of their own CTA: an arrival with release at cluster scope waits for the
  // stores of the warp to be performed, which after an item's output took 2000 cycles.
  // Whether item k may be chosen yet:
  __device__ __forceinline__ bool may_choose(int k) const {
    const int s = k % kItemSlots, n = k / kItemSlots - 1;
    return k < kItemSlots || (wait(L::kItemEmpty + s, n, 81) && wait(L::kItemPeer + s, n, 83) &&
                              mbar_try_wait_acquire_cluster(bar(L::kItemPeer + s), static_cast<uint32_t>(n) & 1u));
  }
  __device__ __forceinline__ uint32_t slot_of(int k) const { return base + L::kItemRing + 48u * static_cast<uint32_t>(k % kItemSlots); }
  __device__ __forceinline__ void publish(int k, const Item& item) const {
    const int s = k % kItemSlots;
    const uint32_t at = slot_of(k), to = mapa_shared(at, 1);
    const uint4 x = make_uint4(item.head, item.row0, item.rows, item.nt), y = make_uint4(item.v[0], item.v[1], item.v[2], item.v[3]);
    const uint4 z = make_uint4(item.v[4], 0, 0, 0);
    st_shared_v4(at, x);
    st_shared_v4(at + 16, y);
    st_shared_v4(at + 32, z);
    mbar_arrive(bar(L::kItemFull + s));
    st_cluster_v4(to, x);
    st_cluster_v4(to + 16, y);
    st_cluster_v4(to + 32, z);
    mbar_arrive_release_cluster(mapa_shared(bar(L::kItemIn + s), 1));
  }
  __device__ __forceinline__ void relay() const {  // the follower's item warp (one lane)
    for (int k = 0;; ++k) {
      const int s = k % kItemSlots, n = k / kItemSlots;
      if (!wait(L::kItemIn + s, n, 82) || !mbar_try_wait_acquire_cluster(bar(L::kItemIn + s), static_cast<uint32_t>(n) & 1u)) return;
      const int head = static_cast<int>(ld_shared_v4(slot_of(k)).x);
      mbar_arrive(bar(L::kItemFull + s));
      if (head < 0) return;
      if (k == 0) continue;
      // (the item before: a warp may be done with it only when it has seen this one)
      const int before = (k - 1) % kItemSlots;
      if (!wait(L::kItemEmpty + before, (k - 1) / kItemSlots, 84)) return;
      mbar_arrive_release_cluster(lbar(L::kItemPeer + before));
    }
  }
  // The other warps wait for item k (all lanes, or one alone), read it, and release it (one lane).
  __device__ __forceinline__ bool await(int k, bool whole_warp) const {
    const bool ok = wait(L::kItemFull + k % kItemSlots, k / kItemSlots, 85);
    return whole_warp ? __all_sync(0xffffffffu, ok) : ok;
  }
  __device__ __forceinline__ Item read(int k) const {
    const uint32_t at = slot_of(k);
    const uint4 a = ld_shared_v4(at), b = ld_shared_v4(at + 16), d = ld_shared_v4(at + 32);
    Item t;
    t.head = static_cast<int>(a.x), t.row0 = static_cast<int>(a.y), t.rows = static_cast<int>(a.z), t.nt = static_cast<int>(a.w);
    t.v[0] = static_cast<int>(b.x), t.v[1] = static_cast<int>(b.y), t.v[2] = static_cast<int>(b.z), t.v[3] = static_cast<int>(b.w);
    t.v[4] = static_cast<int>(d.x);
    return t;
  }
  __device__ __forceinline__ void release(int k) const { mbar_arrive(bar(L::kItemEmpty + k % kItemSlots)); }
};
// The item that the leader chooses as its k-th: its cluster's index first, then the
// next of the list (a counter that the pass over the outputs has set to zero), or
// every n_clusters-th without a counter.
__device__ __forceinline__ int64_t choose_item(int* work, int k, int cluster, int n_clusters) {
  return k == 0 ? cluster : work ? static_cast<int64_t>(n_clusters) + atomicAdd(work, 1) : cluster + static_cast<int64_t>(k) * n_clusters;
}

// Returns false where the block has to leave (both CTAs of the pair alike).  says: this is
// the queries kernel, which leaves its ticket behind its wait; late: the keys kernel behind
// it (BwdArgs::behind_queries), whose wait is at its end when it finds the ticket.
template <typename L>
__device__ __forceinline__ bool enter(Cta<L>& c, uint8_t* smem, const BwdArgs& a, const BwdMaps& maps, bool says, bool late) {
  const uint32_t raw = smem_u32(smem);
  c.base = (raw + 1023u) & ~1023u;
  c.ptr = smem + (c.base - raw);
  c.rank = cluster_ctarank();
  c.leader = c.rank == 0;
  c.warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
  c.lane = threadIdx.x & 31;
  if (c.base - raw + L::kUsed > L::kDynamic) {
    if (threadIdx.x == 0) tc::report_timeout(a.status, 98);
    if (late) grid_dependency_wait();
    return false;
  }
  volatile int* abort_flag = reinterpret_cast<volatile int*>(c.ptr + L::kAbort);
  uint32_t* holder = reinterpret_cast<uint32_t*>(c.ptr + L::kTmemHolder);
  if (threadIdx.x == 0) {
    for (int i = 0; i < L::kNumBars; ++i) {
      const bool scores = i >= L::kSHalf && i <= L::kAccFree;  // the score warps of both CTAs
      const bool local = (i >= L::kStatEmpty && i < L::kItemFull) || (L::kXSlots == 2 && i >= L::kXEmpty && i < L::kYEmpty);  // of this CTA
      const bool items = i >= L::kItemEmpty && i < L::kItemIn;
      mbar_init(c.bar(i), scores ? 2 * kScoreWarps : local ? kScoreWarps : items ? L::kItemTakers + (c.leader ? 1 : 0) : 1);
    }
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (c.warp == kProducerWarp && c.lane == 0 && a.rows > 0) {  // (without query rows there are no maps)
    prefetch_tmap(&maps.q);
    prefetch_tmap(&maps.d_o);
    prefetch_tmap(&maps.ka);
    prefetch_tmap(&maps.va);
    prefetch_tmap(&maps.cols0);
    prefetch_tmap(&maps.cols1);
  }
  if (c.warp == kMmaWarp) {
    tmem_alloc_pair(smem_u32(holder), tc::kTmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  const bool passed = __syncthreads_or(late && threadIdx.x == 0 && ld_acquire_gpu(a.passed) == a.ticket) != 0;
  cluster_sync();
  tc_fence_after();
  c.ctl = Ctl{abort_flag, a.timeout_ns, a.status};
  if (passed)
    fence_proxy_async_global();
  else
    grid_dependency_wait();
  if (threadIdx.x == 0) {
    if (says && blockIdx.x == 0) st_release_gpu(a.passed, a.ticket);
    grid_launch_dependents();
  }
  c.tmem = __shfl_sync(0xffffffffu, *holder, 0);
  return true;
}

// 128 rows from y on (this CTA's part of an operand that is kept).
template <int D>
__device__ __forceinline__ void load_own(uint32_t dst, const CUtensorMap* m, uint32_t full, int x, int y) {
#pragma unroll
  for (int ch = 0; ch < D / 64; ++ch)
#pragma unroll
    for (int h = 0; h < 2; ++h) tma_load_2d_pair(dst + ch * 16384u + h * 8192u, m, full, x + 64 * ch, y + 64 * h);
}
template <int D>
__device__ __forceinline__ void load_half(uint32_t dst, const CUtensorMap* m, uint32_t full, int x, int y) {
#pragma unroll
  for (int ch = 0; ch < D / 64; ++ch) tma_load_2d_pair(dst + ch * 8192u, m, full, x + 64 * ch, y);
}

// Loads that a CTA's producer has issued, by ring: X, Y, rows of S, rows of dP, columns.
struct Loads {
  int n[5] = {0, 0, 0, 0, 0};
  int left;  // until the producer stops: all of them, but for fault injection
  __device__ __forceinline__ Loads(int stop, bool keys, uint32_t rank) {
    left = stop != 0 && ((stop >> 8) & 1) == (keys ? 1 : 0) && static_cast<uint32_t>((stop >> 9) & 1) == rank ? (stop & 255) - 1 : 0x7fffffff;
  }
};

// Teardown, after the roles (`loads` of the producer's lane 0).  As in
// attn_tc2_kernel: when neither CTA gave up, every load was waited for by the MMAs
// that read it; else the leader arms or counts what the other CTA's half lacks,
// and waits for the last phase of each barrier.
template <typename L>
__device__ __forceinline__ void leave(const Cta<L>& c, const Loads& loads) {
  if (c.warp == kProducerWarp && c.lane == 0) {
#pragma unroll
    for (int i = 0; i < 5; ++i) st_cluster_u32(mapa_shared(c.base + L::kLoadRec + 20u * c.rank + 4u * i, 0), static_cast<uint32_t>(loads.n[i]));
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0)
    st_cluster_u32(mapa_shared(c.base + L::kPeerAbort, c.rank ^ 1u), static_cast<uint32_t>(*c.ctl.abort_flag));
  cluster_sync();
  if (c.warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc_pair(c.tmem, tc::kTmemCols);
  }
  if (*c.ctl.abort_flag == 0 && *reinterpret_cast<const volatile int*>(c.ptr + L::kPeerAbort) == 0) return;
  if (c.leader && c.warp == kProducerWarp && c.lane == 0) {
    const volatile uint32_t* mine = reinterpret_cast<const volatile uint32_t*>(c.ptr + L::kLoadRec);
    // bytes: one CTA's of a load
    auto settle = [&](int first, int ring, int slots, uint32_t bytes) {
#pragma unroll 1
      for (int slot = 0; slot < slots; ++slot) {
        auto count = [&](uint32_t total) { return (static_cast<int>(total) - slot + slots - 1) / slots; };
        int m = count(mine[ring]);
        const int theirs = count(mine[5 + ring]);
        if (theirs == m + 1) {
          mbar_arrive_expect_tx(c.bar(first + slot), bytes);
          m = theirs;
        } else if (m == theirs + 1) {
          mbar_complete_tx(c.bar(first + slot), bytes);
        }
        if (m > 0) tc::drain_one(c.bar(first + slot), static_cast<uint32_t>(m - 1) & 1u, c.ctl.timeout_ns);
      }
    };
    settle(L::kXFull, 0, L::kXSlots, L::kXBytes);
    settle(L::kYFull, 1, L::kYLoads, L::kOwn);
    settle(L::kR1Full, 2, L::kSlots, L::kR1Bytes);
    settle(L::kR2Full, 3, L::kR2Loads, L::kHalf);
    settle(L::kCFull, 4, L::kSlots, L::kCBytes);
  }
  cluster_sync();
}

// The producer's next load of a ring: waits until its slot is free and arms the
// barrier (leader); the slot, or -1 when it gave up.
template <typename L>
__device__ __forceinline__ int begin_load(const Cta<L>& c, Loads& loads, int ring, int slots, int full, int empty, uint32_t bytes, int where) {
  const int n = loads.n[ring], slot = n % slots;
  if (loads.left == 0) return -1;
  if (n >= slots && !c.wait(empty + slot, n / slots - 1, where)) return -1;
  if (c.leader) mbar_arrive_expect_tx(c.bar(full + slot), 2 * bytes);
  ++loads.n[ring];
  --loads.left;
  return slot;
}
}  // namespace bwd

// kRef32: the cached rows' gradients are fp32, here and in what is added (BwdArgs).
template <int D, bool kRef32>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(bwd::kThreads, 1)
    attn_bwd_keys_kernel(const __grid_constant__ BwdMaps maps, const __grid_constant__ BwdKeys keys, const __grid_constant__ BwdArgs args) {
  using namespace bwd;
  using L = Smem<D, true>;
  constexpr int kAhead = L::kSBufs;  // tiles that S is ahead of dV
  constexpr uint32_t kColS = 0, kColP = 128 * kAhead, kColV = kColP + 128, kColK = kColV + D;
  static_assert(kColK + D <= tc::kTmemCols, "tensor-memory layout");
  extern __shared__ uint8_t smem_raw[];
  Cta<L> c;
  if (!enter(c, smem_raw, args, maps, false, args.behind_queries != 0)) return;
  const int cluster = static_cast<int>(blockIdx.x >> 1), n_clusters = static_cast<int>(gridDim.x >> 1);
  const int n_items = keys.n_tiles * args.num_heads;
  Loads loads(args.dbg_stop, true, c.rank);
  if (c.warp == kProducerWarp) {
    if (c.lane == 0) {
      int s = 0;
#pragma unroll 1
      for (int k = 0; s >= 0 && c.await(k, false); ++k) {
        const Item t = c.read(k);
        c.release(k);
        if (t.head < 0) break;
        if (t.nt == 0) continue;
        const int x = t.head * D, xc = x + D / 2 * static_cast<int>(c.rank), r64 = 64 * static_cast<int>(c.rank);
        const int y = t.row0 + 128 * static_cast<int>(c.rank);
        if ((s = begin_load(c, loads, 0, 1, L::kXFull, L::kXEmpty, L::kXBytes, 31)) < 0) break;
        load_own<D>(c.base + L::kX, t.v[2] ? &maps.kb : &maps.ka, c.lbar(L::kXFull), x, y);
        load_own<D>(c.base + L::kY, t.v[2] ? &maps.vb : &maps.va, c.lbar(L::kXFull), x, y);
#pragma unroll 1
        for (int j = 0; j < t.nt; ++j) {
          const int y0 = t.v[0] + kTile * j;
          if ((s = begin_load(c, loads, 2, L::kSlots, L::kR1Full, L::kR1Empty, L::kR1Bytes, 32)) < 0) break;
          const uint32_t r = c.base + L::kR1 + s * L::kR1Bytes;
          load_half<D>(r, &maps.q, c.lbar(L::kR1Full + s), x, y0 + r64);
          load_half<D>(r + L::kHalf, &maps.d_o, c.lbar(L::kR1Full + s), x, y0 + r64);
          if ((s = begin_load(c, loads, 4, L::kSlots, L::kCFull, L::kCEmpty, L::kCBytes, 35)) < 0) break;
          const uint32_t d = c.base + L::kC + s * L::kCBytes;
          tma_load_2d_pair(d, &maps.cols0, c.lbar(L::kCFull + s), xc, y0);
          tma_load_2d_pair(d + L::kHalf, &maps.cols1, c.lbar(L::kCFull + s), xc, y0);
        }
      }
    }
    __syncwarp();
  } else if (c.warp == kItemWarp) {
    if (c.leader && c.lane == 0) {
      // Kept apart from the producer, whose loads are few tiles ahead: choosing, decoding
      // and passing on an item takes longer than that.  An item is chosen while the one
      // before it runs, not earlier: a pair that holds more leaves others idle at the end.
      auto item_of = [&](int64_t it) -> Item {
        Item t{};
        t.head = -1;
        if (it >= n_items) return t;
        const BwdItem i = bwd_item(keys, static_cast<int>(it), args.num_heads);
        const BwdKeySeg& s = keys.seg[i.seg];
        const int r0 = i.tile * kBlock;
        t.head = i.head;
        t.row0 = s.k_row0 + r0;
        t.rows = min(kBlock, s.k_rows - r0);
        t.nt = (s.q_rows + kTile - 1) / kTile;
        t.v[0] = s.q_row0, t.v[1] = s.q_rows, t.v[2] = s.in_b;
        t.v[3] = s.add_from - r0, t.v[4] = s.add_row0 + r0;  // within the item
        return t;
      };
      for (int k = 0; c.may_choose(k); ++k) {
        const Item t = item_of(choose_item(args.work_keys, k, cluster, n_clusters));
        c.publish(k, t);
        if (t.head < 0) break;
      }
    } else if (c.lane == 0) {
      c.relay();
    }
    __syncwarp();
  } else if (c.warp == kMmaWarp) {
    if (c.leader) {
      const uint64_t xd = sdesc_sw128(c.base + L::kX, 16, 1024), yd = sdesc_sw128(c.base + L::kY, 16, 1024);
      const uint64_t rd = sdesc_sw128(c.base + L::kR1, 16, 1024), cd = cols_desc<D>(c.base + L::kC);
      const uint32_t tm = c.tmem;
      bool issued = false;
      int t = 0, n = 0;  // tiles, and items with tiles, so far
      auto rows = [&](int i) { return rd + static_cast<uint64_t>(i % L::kSlots) * (L::kR1Bytes >> 4); };
      auto rows_ready = [&](int i) { return c.wait_all(L::kR1Full + i % L::kSlots, i / L::kSlots, 37); };
      auto issue_s = [&](int i) {
        mma_rows<D>(tm + kColS + 128u * (i % kAhead), xd, rows(i));
        tc2_commit_mc(c.bar(L::kSDone + i % kAhead), 3);
      };
      // (dP's commit also frees the tile's rows and, with the last tile, the item's own)
      auto issue_dp = [&](int i, bool last) {
        mma_rows<D>(tm + kColP, yd, rows(i) + (L::kHalf >> 4));
        tc2_commit_mc(c.bar(L::kPDone), 3);
        tc2_commit_mc(c.bar(L::kR1Empty + i % L::kSlots), 3);
        if (last) tc2_commit_mc(c.bar(L::kXEmpty), 3);
      };
#pragma unroll 1
      for (int k = 0;; ++k) {
        if (!c.await(k, true)) goto mma_done;
        const int head = __shfl_sync(0xffffffffu, c.read(k).head, 0), nt = __shfl_sync(0xffffffffu, c.read(k).nt, 0);
        __syncwarp();
        if (c.lane == 0) c.release(k);
        if (head < 0) break;
        if (nt == 0) continue;
        if (!c.wait_all(L::kXFull, n, 36) || !rows_ready(t)) goto mma_done;
        issued = true;
        if (elect_one()) {
          tc_fence_after();
          issue_s(t);
          issue_dp(t, nt == 1);
        }
        __syncwarp();
        if (kAhead == 2 && nt > 1) {
          if (!rows_ready(t + 1)) goto mma_done;
          if (elect_one()) {
            tc_fence_after();
            issue_s(t + 1);
          }
          __syncwarp();
        }
#pragma unroll 1
        for (int j = 0; j < nt; ++j, ++t) {
          const bool next = j + 1 < nt;
          const uint64_t cols = cd + static_cast<uint64_t>(t % L::kSlots) * (L::kCBytes >> 4);
          if (!c.wait_all(L::kCFull + t % L::kSlots, t / L::kSlots, 40)) goto mma_done;
          if (j == 0 && n > 0 && !c.wait_all(L::kAccFree, n - 1, 41)) goto mma_done;
          const bool s_next = j + kAhead < nt;
          if (s_next && !rows_ready(t + kAhead)) goto mma_done;
          const uint32_t t_p = tm + kColS + 128u * (t % kAhead), acc = j > 0 ? 1u : 0u;
          if (kAhead == 1) {  // the first half of P
            if (!c.wait_all(L::kSHalf, t, 49)) goto mma_done;
            if (elect_one()) {
              tc_fence_after();
              mma_cols<D, 0>(tm + kColV, t_p, cols, acc);
            }
            __syncwarp();
          }
          if (!c.wait_all(L::kSUsed + t % kAhead, t / kAhead, 42)) goto mma_done;  // P is written
          if (elect_one()) {
            tc_fence_after();
            mma_cols<D, kAhead == 1 ? 1 : -1>(tm + kColV, t_p, cols, acc);
            if (s_next) issue_s(t + kAhead);
          }
          __syncwarp();
          if (!c.wait_all(L::kDsFull, t, 43)) goto mma_done;
          if (elect_one()) {
            tc_fence_after();
            mma_cols<D, -1>(tm + kColK, tm + kColP, cols + (L::kHalf >> 4), j > 0 ? 1u : 0u);
            tc2_commit_mc(c.bar(L::kCEmpty + t % L::kSlots), 3);
            if (next)
              issue_dp(t + 1, j + 2 == nt);
            else
              tc2_commit_mc(c.bar(L::kAccDone), 3);
          }
          __syncwarp();
        }
        ++n;
      }
    mma_done:
      __syncwarp();
      if (issued && elect_one()) {
        tc2_commit_mc(c.bar(L::kMmaDone), 1);
        tc::drain_one(c.bar(L::kMmaDone), 0u, args.timeout_ns);
      }
    }
    __syncwarp();
  } else if (c.warp == kStatWarp) {
    // (-lse log2 e, -delta) of each query of a tile, two arrays of 128; rows past the end get P = 0
    int t = 0;
    bool ok = true;
#pragma unroll 1
    for (int k = 0; ok && c.await(k, true); ++k) {
      const Item m = c.read(k);
      __syncwarp();
      if (c.lane == 0) c.release(k);
      if (m.head < 0) break;
      const float2* src = args.stats + m.head * args.rows + m.v[0];
#pragma unroll 1
      for (int j = 0; j < m.nt; ++j, ++t) {
        float2 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = kTile * j + 32 * i + c.lane;
          v[i] = r < m.v[1] ? src[r] : make_float2(INFINITY, 0.f);
        }
        const int s = t % kStatSlots;
        if (t >= kStatSlots && !(ok = c.wait_all(L::kStatEmpty + s, t / kStatSlots - 1, 48))) break;
        float* dst = reinterpret_cast<float*>(c.ptr + L::kStat + 1024 * s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          dst[32 * i + c.lane] = -v[i].x;
          dst[128 + 32 * i + c.lane] = -v[i].y;
        }
        __syncwarp();
        if (c.lane == 0) mbar_arrive(c.bar(L::kStatFull + s));
      }
    }
  } else {
    const int half = c.warp >> 2, lane0 = 32 * (c.warp & 3);
    const int row = 128 * static_cast<int>(c.rank) + lane0;  // the warp's first row in an item
    const uint32_t lanes = static_cast<uint32_t>(lane0) << 16;
    const uint32_t t_p = c.tmem + lanes + kColP + 64 * half;
    const f32x2 sl2 = make_f32x2(args.scale_log2, args.scale_log2);
    const uint32_t l_bars = c.lbar(0);
    auto arrive = [&](int b) {
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (c.lane == 0) mbar_arrive_cluster(l_bars + 8u * static_cast<uint32_t>(b));
    };
    // dV (warps 0-3) and dK (warps 4-7) of this warp's 32 keys for the n-th item with tiles
    auto write_out = [&](const Item& m, int n) -> bool {
      const float scale = half ? args.scale : 1.f;
      const int64_t at = (static_cast<int64_t>(m.row0) + row) * args.row_stride + m.head * D;
      using Ref = std::conditional_t<kRef32, float, __nv_bfloat16>;
      void* const ref = half ? args.dkb : args.dvb;
      __nv_bfloat16* const out = (m.v[2] ? static_cast<__nv_bfloat16*>(ref) : half ? args.dka : args.dva) + at;
      const int first = m.v[3] - row, rows = m.rows - row;  // of the warp's rows: from `first` on something is added
      const bool adds = first < min(32, rows);
      const Ref* add = static_cast<const Ref*>(half ? args.add_k : args.add_v) + (static_cast<int64_t>(m.v[4]) + row) * args.row_stride + m.head * D;
      const RowsOut stage{c.base + L::kStage + 4096u * c.warp, c.lane};
      // (in whole lines through the stage, before the wait: from the registers, 16 bytes of
      // each of 32 rows at a time, it took 4000 cycles of an item)
      if (adds) stage.fetch(add, args.row_stride, first, rows);
      if (!c.wait_all(L::kAccDone, n, 47)) return false;
      tc_fence_after();
#pragma unroll
      for (int cc = 0; cc < D / 64; ++cc) {
        if (cc > 0 && adds) stage.fetch(add + 64 * cc, args.row_stride, first, rows);
        float v[64];
        load64(c.tmem + lanes + (half ? kColK : kColV) + 64 * cc, v);
        if (cc + 1 == D / 64) {  // all of it is read
          tc_fence_before();
          __syncwarp();
          if (c.lane == 0) mbar_arrive_cluster(l_bars + 8u * L::kAccFree);
        }
        if constexpr (kRef32) {  // 32 columns at a time
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if (s > 0 && adds) {
              __syncwarp();
              stage.fetch(add + 64 * cc + 32, args.row_stride, first, rows);
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const uint4 y = adds ? stage.get(q) : make_uint4(0, 0, 0, 0);  // (zeros where nothing is added)
              float* x = v + 32 * s + 4 * q;
              const uint32_t add4[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
              for (int e = 0; e < 4; ++e)  // (the product rounded by itself, as below: the same sums as with bf16)
                x[e] = __fadd_rn(__fmul_rn(x[e], scale), __uint_as_float(add4[e]));
            }
          }
          __syncwarp();
          if (m.v[2]) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
#pragma unroll
              for (int q = 0; q < 8; ++q) {
                const float* x = v + 32 * s + 4 * q;
                stage.put(q, make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])));
              }
              stage.flush(static_cast<float*>(ref) + at + 64 * cc + 32 * s, args.row_stride, rows);
            }
            continue;
          }
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          Vec8 x;
#pragma unroll
          for (int e = 0; e < 8; ++e) x.v[e] = kRef32 ? v[8 * q + e] : v[8 * q + e] * scale;
          if (!kRef32 && adds) {
            const Vec8 y = unpack8(stage.get(q));
#pragma unroll
            for (int e = 0; e < 8; ++e) x.v[e] += y.v[e];
          }
          stage.put(q, pack8(x));
        }
        stage.flush(out + 64 * cc, args.row_stride, rows);
      }
      return true;
    };
    // The gradients of an item that no query sees: zero, or what is added to them.
    auto write_none = [&](const Item& m) {
      const int r = row + c.lane;
      if (r >= m.rows) return;
      const int64_t at = (static_cast<int64_t>(m.row0) + r) * args.row_stride + m.head * D;
      const int64_t from = (static_cast<int64_t>(m.v[4]) + r) * args.row_stride + m.head * D;
      auto write = [&](auto* out, const auto* add) {
        constexpr int kPer = 16 / sizeof(*out);
#pragma unroll 1
        for (int i = 0; i < D; i += kPer)
          *reinterpret_cast<uint4*>(out + i) = r >= m.v[3] ? *reinterpret_cast<const uint4*>(add + i) : make_uint4(0, 0, 0, 0);
      };
      // (the call's own keys, which the call's own queries see, are never of such an item)
      using Ref = std::conditional_t<kRef32, float, __nv_bfloat16>;
      write(static_cast<Ref*>(half ? args.dkb : args.dvb) + at, static_cast<const Ref*>(half ? args.add_k : args.add_v) + from);
    };
    int t = 0, n = 0;  // tiles, and items with tiles, so far
#pragma unroll 1
    for (int k = 0;; ++k) {
      if (!c.await(k, true)) goto scores_done;
      const Item m = c.read(k);
      if (m.head < 0) break;
      if (m.nt == 0) {
        write_none(m);
        __syncwarp();
        if (c.lane == 0) c.release(k);
        continue;
      }
      bool ready = false;  // this tile's S and statistics were seen at the end of the tile before
#pragma unroll 1
      for (int j = 0; j < m.nt; ++j, ++t) {
        const int s = t % kStatSlots;
        const uint32_t stat = c.base + L::kStat + 1024u * s + 256u * half;
        const uint32_t t_s = c.tmem + lanes + kColS + 128u * (t % kAhead) + 64u * half;
        float p[64];
        if (!ready && (!c.wait_all(L::kStatFull + s, t / kStatSlots, 44) || !c.wait_all(L::kSDone + t % kAhead, t / kAhead, 45))) goto scores_done;
        tc_fence_after();
        {
          uint32_t r[2][32];
          tmem_ld32(t_s, r[0]);
          tmem_wait_ld(r[0]);
          tmem_ld32(t_s + 32, r[1]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (h == 1) tmem_wait_ld(r[1]);
            uint32_t pk[16];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const float4 nl = ld_shared_f4(stat + 128u * h + 16u * q);
              const uint32_t* x = r[h] + 4 * q;
              float* y = p + 32 * h + 4 * q;
              float e0, e1, e2, e3;
              split_f32x2(fma_f32x2(make_f32x2(__uint_as_float(x[0]), __uint_as_float(x[1])), sl2, make_f32x2(nl.x, nl.y)), e0, e1);
              split_f32x2(fma_f32x2(make_f32x2(__uint_as_float(x[2]), __uint_as_float(x[3])), sl2, make_f32x2(nl.z, nl.w)), e2, e3);
              y[0] = ex2_approx(e0), y[1] = ex2_approx(e1), y[2] = ex2_approx(e2), y[3] = ex2_approx(e3);
              pk[2 * q] = pack_bf16x2(y[0], y[1]);
              pk[2 * q + 1] = pack_bf16x2(y[2], y[3]);
            }
            // (over the first 32 columns read, which both halves fit in)
            tmem_st16(t_s + 16u * h, pk);
            if (kAhead == 1 && h == 0) arrive(L::kSHalf);
          }
        }
        arrive(L::kSUsed + t % kAhead);
        if (!c.wait_all(L::kPDone, t, 46)) goto scores_done;
        tc_fence_after();
        {
          uint32_t r[2][32];
          tmem_ld32(t_p, r[0]);
          tmem_wait_ld(r[0]);
          tmem_ld32(t_p + 32, r[1]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (h == 1) tmem_wait_ld(r[1]);
            uint32_t pk[16];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const float4 ndl = ld_shared_f4(stat + 512u + 128u * h + 16u * q);
              const uint32_t* d = r[h] + 4 * q;
              const float* y = p + 32 * h + 4 * q;
              float e0, e1, e2, e3;
              split_f32x2(mul_f32x2(make_f32x2(y[0], y[1]),
                                    add_f32x2(make_f32x2(__uint_as_float(d[0]), __uint_as_float(d[1])), make_f32x2(ndl.x, ndl.y))), e0, e1);
              split_f32x2(mul_f32x2(make_f32x2(y[2], y[3]),
                                    add_f32x2(make_f32x2(__uint_as_float(d[2]), __uint_as_float(d[3])), make_f32x2(ndl.z, ndl.w))), e2, e3);
              pk[2 * q] = pack_bf16x2(e0, e1);
              pk[2 * q + 1] = pack_bf16x2(e2, e3);
            }
            tmem_st16(t_p + 16u * h, pk);
          }
        }
        // a look at the next tile, whose latency passes beside the stores
        const int u = t + 1;
        const bool next = j + 1 < m.nt && c.done(L::kStatFull + u % kStatSlots, u / kStatSlots) && c.done(L::kSDone + u % kAhead, u / kAhead);
        arrive(L::kDsFull);
        ready = __all_sync(0xffffffffu, next);
        if (c.lane == 0) mbar_arrive(c.bar(L::kStatEmpty + s));
      }
      __syncwarp();
      if (c.lane == 0) c.release(k);
      if (!write_out(m, n)) goto scores_done;
      ++n;
    }
  scores_done:;
  }
  leave(c, loads);
  if (args.behind_queries) {
    grid_dependency_wait();  // the work after this kernel sees both
    // (a CTA that starts later and finds no ticket waits for nothing any more)
    if (blockIdx.x == 0 && threadIdx.x == 0) st_release_gpu(args.passed, 0);
  }
}

template <int D>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(bwd::kThreads, 1)
    attn_bwd_queries_kernel(const __grid_constant__ BwdMaps maps, const __grid_constant__ BwdQueries queries,
                            const __grid_constant__ BwdArgs args) {
  using namespace bwd;
  using L = Smem<D, false>;
  constexpr uint32_t kColS = 0, kColP = 128, kColQ = 384;
  extern __shared__ uint8_t smem_raw[];
  Cta<L> c;
  if (!enter(c, smem_raw, args, maps, true, false)) return;
  const int cluster = static_cast<int>(blockIdx.x >> 1), n_clusters = static_cast<int>(gridDim.x >> 1);
  const int n_items = queries.n_tiles * args.num_heads;
  Loads loads(args.dbg_stop, false, c.rank);
  if (c.warp == kProducerWarp) {
    if (c.lane == 0) {
      Item t{}, next{};
      int s = 0;
      bool x_loaded = false, c_due = false, c_b = false;  // columns of the tile before, whose dQ comes a tile later
      int c_x = 0, c_y = 0;
      auto load_x = [&](const Item& m) -> bool {
        const int b = begin_load(c, loads, 0, L::kXSlots, L::kXFull, L::kXEmpty, L::kOwn, 51);
        if (b < 0) return false;
        load_own<D>(c.base + L::kX + b * L::kXSlot, &maps.q, c.lbar(L::kXFull + b), m.head * D, m.row0 + 128 * static_cast<int>(c.rank));
        return true;
      };
      auto load_cols = [&]() -> bool {
        const int b = begin_load(c, loads, 4, L::kSlots, L::kCFull, L::kCEmpty, L::kCBytes, 55);
        if (b < 0) return false;
        tma_load_2d_pair(c.base + L::kC + b * L::kCBytes, c_b ? &maps.cols1 : &maps.cols0, c.lbar(L::kCFull + b), c_x, c_y);
        return true;
      };
      auto get_next = [&](int k) -> bool {  // the item after item k
        if (!c.await(k + 1, false)) return false;
        next = c.read(k + 1);
        c.release(k + 1);
        return true;
      };
      bool ok = get_next(-1);
#pragma unroll 1
      for (int k = 0; ok && next.head >= 0; ++k) {
        t = next;
        const int x = t.head * D, xc = x + D / 2 * static_cast<int>(c.rank), r64 = 64 * static_cast<int>(c.rank);
        if (!x_loaded && !(ok = load_x(t))) break;
        x_loaded = false;
#pragma unroll 1
        for (int j = 0; ok && j < t.nt; ++j) {
          const bool b = j >= t.v[4];
          const int y0 = b ? t.v[2] + kTile * (j - t.v[4]) : t.v[0] + kTile * j;
          ok = false;
          if ((s = begin_load(c, loads, 2, L::kSlots, L::kR1Full, L::kR1Empty, L::kR1Bytes, 52)) < 0) break;
          load_half<D>(c.base + L::kR1 + s * L::kR1Bytes, b ? &maps.kb : &maps.ka, c.lbar(L::kR1Full + s), x, y0 + r64);
          if (!L::kRApart) load_half<D>(c.base + L::kR1 + s * L::kR1Bytes + L::kHalf, b ? &maps.vb : &maps.va, c.lbar(L::kR1Full + s), x, y0 + r64);
          if (j == 0) {
            if ((s = begin_load(c, loads, 1, L::kYSlots, L::kYFull, L::kYEmpty, L::kOwn, 53)) < 0) break;
            load_own<D>(c.base + L::kY + s * L::kOwn, &maps.d_o, c.lbar(L::kYFull + s), x, t.row0 + 128 * static_cast<int>(c.rank));
          }
          if (L::kRApart) {
            if ((s = begin_load(c, loads, 3, L::kSlots, L::kR2Full, L::kR2Empty, L::kHalf, 54)) < 0) break;
            load_half<D>(c.base + L::kR2 + s * L::kHalf, b ? &maps.vb : &maps.va, c.lbar(L::kR2Full + s), x, y0 + r64);
          }
          if (c_due && !load_cols()) break;
          c_due = true, c_b = b, c_x = xc, c_y = y0;
          if (j == max(0, t.nt - 3)) {  // the next item's X, ahead of this one's last tiles
            if (!get_next(k)) break;
            if (next.head >= 0) {
              if (!load_x(next)) break;
              x_loaded = true;
            }
          }
          ok = true;
        }
      }
      if (ok && c_due) load_cols();
    }
    __syncwarp();
  } else if (c.warp == kItemWarp) {
    if (c.leader && c.lane == 0) {
      // Kept apart from the producer, whose loads are few tiles ahead: choosing, decoding
      // and passing on an item takes longer than that.  An item is chosen while the one
      // before it runs, not earlier: a pair that holds more leaves others idle at the end.
      auto item_of = [&](int64_t it) -> Item {
        Item t{};
        t.head = -1;
        if (it >= n_items) return t;
        const BwdItem i = bwd_item(queries, static_cast<int>(it), args.num_heads);
        const BwdQuerySeg& s = queries.seg[i.seg];
        const int r0 = i.tile * kBlock;
        t.head = i.head;
        t.row0 = s.q_row0 + r0;
        t.rows = min(kBlock, s.q_rows - r0);
        t.v[0] = s.a_row0, t.v[1] = s.a_len, t.v[2] = s.b_row0, t.v[3] = s.b_len;
        t.v[4] = (s.a_len + kTile - 1) / kTile;
        t.nt = t.v[4] + (s.b_len + kTile - 1) / kTile;
        return t;
      };
      for (int k = 0; c.may_choose(k); ++k) {
        const Item t = item_of(choose_item(args.work_queries, k, cluster, n_clusters));
        c.publish(k, t);
        if (t.head < 0) break;
      }
    } else if (c.lane == 0) {
      c.relay();
    }
    __syncwarp();
  } else if (c.warp == kMmaWarp) {
    if (c.leader) {
      const uint64_t xd = sdesc_sw128(c.base + L::kX, 16, 1024), yd = sdesc_sw128(c.base + L::kY, 16, 1024);
      const uint64_t r1 = sdesc_sw128(c.base + L::kR1, 16, 1024), r2 = sdesc_sw128(c.base + L::kR2, 16, 1024);
      const uint64_t cd = cols_desc<D>(c.base + L::kC);
      const uint32_t tm = c.tmem;
      bool issued = false;
      int nt = 0, k = -1, j = 0;  // S and dP: tile j of nt of item k
      int pj = 0, pnt = 0, pk = 0;  // dQ, a tile behind: tile pj of pnt of item pk
      // step t: S and dP of tile t, then dQ of tile t - 1
#pragma unroll 1
      for (int t = 0;; ++t) {
        if (j == nt) {
          ++k;
          if (!c.await(k, true)) goto mma_done;
          nt = __shfl_sync(0xffffffffu, c.read(k).nt, 0);  // (0 where none is left)
          __syncwarp();
          if (c.lane == 0) c.release(k);
          j = 0;
        }
        if (nt > 0) {
          const int u = t & 1, r = t % L::kSlots, h = t / L::kSlots;
          const uint64_t kb = static_cast<uint64_t>(k & 1);
          if (j == 0 && !c.wait_all(L::kXFull + (k & 1), k >> 1, 56)) goto mma_done;
          if (!c.wait_all(L::kR1Full + r, h, 57)) goto mma_done;
          if (t > 0 && !c.wait_all(L::kSUsed, t - 1, 58)) goto mma_done;
          if (!L::kRApart && j == 0 && !c.wait_all(L::kYFull + (k & 1), k >> 1, 59)) goto mma_done;
          issued = true;
          if (elect_one()) {
            tc_fence_after();
            mma_rows<D>(tm + kColS, xd + kb * (L::kXSlot >> 4), r1 + static_cast<uint64_t>(r) * (L::kR1Bytes >> 4));
            tc2_commit_mc(c.bar(L::kSDone), 3);
            if (L::kRApart) tc2_commit_mc(c.bar(L::kR1Empty + r), 3);
            else {
              mma_rows<D>(tm + kColP + 128u * u, yd + kb * (L::kOwn >> 4), r1 + static_cast<uint64_t>(r) * (L::kR1Bytes >> 4) + (L::kHalf >> 4));
              tc2_commit_mc(c.bar(L::kPDone + u), 3);
              tc2_commit_mc(c.bar(L::kR1Empty + r), 3);
              if (j + 1 == nt) tc2_commit_mc(c.bar(L::kYEmpty + (k & 1)), 3);
            }
          }
          __syncwarp();
          if (L::kRApart) {
            if (j == 0 && !c.wait_all(L::kYFull + (k & 1), k >> 1, 59)) goto mma_done;
            if (!c.wait_all(L::kR2Full + r, h, 60)) goto mma_done;
            if (elect_one()) {
              tc_fence_after();
              mma_rows<D>(tm + kColP + 128u * u, yd + kb * (L::kOwn >> 4), r2 + static_cast<uint64_t>(r) * (L::kHalf >> 4));
              tc2_commit_mc(c.bar(L::kPDone + u), 3);
              tc2_commit_mc(c.bar(L::kR2Empty + r), 3);
              if (j + 1 == nt) tc2_commit_mc(c.bar(L::kYEmpty + (k & 1)), 3);
            }
            __syncwarp();
          }
        }
        if (t > 0) {
          const int i = t - 1, u = i & 1, r = i % L::kSlots;
          if (!c.wait_all(L::kCFull + r, i / L::kSlots, 61)) goto mma_done;
          if (pj == 0 && pk > 0 && !c.wait_all(L::kAccFree, pk - 1, 62)) goto mma_done;
          if (!c.wait_all(L::kDsFull + u, i >> 1, 63)) goto mma_done;
          if (elect_one()) {
            tc_fence_after();
            mma_cols<D, -1>(tm + kColQ, tm + kColP + 128u * u, cd + static_cast<uint64_t>(r) * (L::kCBytes >> 4), pj > 0 ? 1u : 0u);
            tc2_commit_mc(c.bar(L::kCEmpty + r), 3);
            if (pj + 1 == pnt) tc2_commit_mc(c.bar(L::kAccDone), 3);
          }
          __syncwarp();
        }
        if (nt == 0) break;
        pj = j, pnt = nt, pk = k;
        ++j;
      }
    mma_done:
      __syncwarp();
      if (issued && elect_one()) {
        tc2_commit_mc(c.bar(L::kMmaDone), 1);
        tc::drain_one(c.bar(L::kMmaDone), 0u, args.timeout_ns);
      }
    }
    __syncwarp();
  } else if (c.warp < kScoreWarps) {
    const int half = c.warp >> 2, lane0 = 32 * (c.warp & 3);
    const uint32_t lanes = static_cast<uint32_t>(lane0) << 16;
    const uint32_t t_s = c.tmem + lanes + kColS + 64 * half, t_p = c.tmem + lanes + kColP + 64 * half;
    const f32x2 sl2 = make_f32x2(args.scale_log2, args.scale_log2);
    const uint32_t l_used = c.lbar(L::kSUsed), l_ds = c.lbar(L::kDsFull), l_free = c.lbar(L::kAccFree);
    const int row = 128 * static_cast<int>(c.rank) + lane0;  // the warp's first row in an item
    // dQ of item k: columns [D / 2 half, D / 2 (half + 1)) of this warp's 32 rows
    auto write_out = [&](int k) -> bool {
      const Item m = c.read(k);
      __syncwarp();
      if (c.lane == 0) c.release(k);
      if (!c.wait_all(L::kAccDone, k, 67)) return false;
      tc_fence_after();
      uint32_t v[D / 2];
      if constexpr (D == 128) {
        uint32_t(&v0)[32] = reinterpret_cast<uint32_t(&)[32]>(v);
        uint32_t(&v1)[32] = reinterpret_cast<uint32_t(&)[32]>(v[32]);
        tmem_ld32(c.tmem + lanes + kColQ + 64u * half, v0);
        tmem_ld32(c.tmem + lanes + kColQ + 64u * half + 32u, v1);
        tmem_wait_ld(v0);
        tmem_wait_ld(v1);
      } else {
        tmem_ld32(c.tmem + lanes + kColQ + 32u * half, v);
        tmem_wait_ld(v);
      }
      tc_fence_before();
      __syncwarp();
      if (c.lane == 0) mbar_arrive_cluster(l_free);
      // staged in the item's Q, which its last S has read: chunks of 16 bytes, eight a row, or four at D = 64
      const RowsOut rows{c.base + L::kX + L::kXSlot * static_cast<uint32_t>(k & 1) + 4096u * c.warp, c.lane};
#pragma unroll
      for (int q = 0; q < D / 16; ++q) {
        Vec8 x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x.v[e] = __uint_as_float(v[8 * q + e]) * args.scale;
        rows.put(q, pack8(x));
      }
      __nv_bfloat16* out = args.dq + (static_cast<int64_t>(m.row0) + row) * args.row_stride + m.head * D + D / 2 * half;
      if constexpr (D == 128) {
        rows.flush(out, args.row_stride, m.rows - row);
      } else {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 8 * i + (c.lane >> 2), ch = c.lane & 3;
          const uint4 x = ld_shared_v4(rows.stage + 128u * r + (static_cast<uint32_t>(ch ^ (r & 7)) << 4));
          if (r < m.rows - row) *reinterpret_cast<uint4*>(out + r * args.row_stride + 8 * ch) = x;
        }
        __syncwarp();
      }
      fence_proxy_async_smem();  // the buffer is free for the loads of the item after the next
      __syncwarp();
      if (c.lane == 0) mbar_arrive(c.bar(L::kXEmpty + (k & 1)));
      return true;
    };
    int t = 0, k = 0;
#pragma unroll 1
    for (;; ++k) {  // item k; the dQ of item k - 1 is written behind its first P
      if (!c.await(k, true)) goto scores_done;
      const Item m = c.read(k);
      if (m.head < 0) {
        __syncwarp();
        if (c.lane == 0) c.release(k);
        break;
      }
      const float2 st = row + c.lane < m.rows ? args.stats[m.head * args.rows + m.row0 + row + c.lane] : make_float2(INFINITY, 0.f);
      const f32x2 nl = make_f32x2(-st.x, -st.x), ndl = make_f32x2(-st.y, -st.y);
#pragma unroll 1
      for (int j = 0; j < m.nt; ++j, ++t) {
        float p[64];
        if (!c.wait_all(L::kSDone, t, 65)) goto scores_done;
        tc_fence_after();
        const int valid = (j < m.v[4] ? m.v[1] - kTile * j : m.v[3] - kTile * (j - m.v[4])) - 64 * half;  // of this warp's 64 keys
        if (valid < 64) {  // keys past the end: scores of -inf
#pragma unroll 1
          for (int i = max(valid, 0); i < 64; ++i) tmem_st1(t_s + static_cast<uint32_t>(i), 0xFF800000u);
          tmem_wait_st();
        }
        load64(t_s, p);
        tc_fence_before();
        __syncwarp();
        if (c.lane == 0) mbar_arrive_cluster(l_used);
#pragma unroll
        for (int i = 0; i < 64; i += 2) {
          float e0, e1;
          split_f32x2(fma_f32x2(make_f32x2(p[i], p[i + 1]), sl2, nl), e0, e1);
          p[i] = ex2_approx(e0), p[i + 1] = ex2_approx(e1);
        }
        if (j == 0 && k > 0 && !write_out(k - 1)) goto scores_done;
        const int b = t & 1;
        if (!c.wait_all(L::kPDone + b, t >> 1, 66)) goto scores_done;
        tc_fence_after();
        {
          float d[64];
          load64(t_p + 128u * b, d);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t pk[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) {
              const int i = 32 * h + 2 * q;
              float e0, e1;
              split_f32x2(mul_f32x2(make_f32x2(p[i], p[i + 1]), add_f32x2(make_f32x2(d[i], d[i + 1]), ndl)), e0, e1);
              pk[q] = pack_bf16x2(e0, e1);
            }
            tmem_st16(t_p + 128u * b + 16u * h, pk);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (c.lane == 0) mbar_arrive_cluster(l_ds + 8u * b);
      }
    }
    if (k > 0) write_out(k - 1);
  scores_done:;
  }
  leave(c, loads);
}

}  // namespace rc
