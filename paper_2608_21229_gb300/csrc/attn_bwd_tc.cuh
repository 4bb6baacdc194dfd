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
// over the rows.  Per tile of 128 x 128 (512 tensor cycles a product at D = 128)
// the tensor core then reads 192 KB (keys kernel) of shared memory in 2048
// cycles, and 64 KB arrive: below the 128 bytes a cycle that an SM's shared memory
// gives, which one CTA alone (M = 128) would need in full.
//
// Tensor memory (512 columns), keys kernel: S^T [0, 128), dP^T [128, 256), dV
// [256, 384), dK [384, 512); P^T and dS^T as bf16 over the scores they come from.
// The tensor core's order of work is
//   S_0 dP_0 | dV_0 S_1 | dK_0 dP_1 | dV_1 S_2 | dK_1 dP_2 | ...
// so that P_i is found from S_i while dK_i-1 and dP_i run, and dS_i from dP_i while
// dV_i and S_i+1 run: each has 1024 tensor cycles, with one buffer each.
// Queries kernel: S [0, 128), dP twice [128, 384), dQ [384, 512); P never leaves
// the registers, S is free as soon as it is read, and the order is
//   S_i dP_i dQ_i-1 | S_i+1 dP_i+1 dQ_i | ...
//
// Warps: 0-7 scores (warp w: lanes 32 (w % 4).., columns 64 (w / 4)..; P and dS are
// written over the columns that the same warp has read), 8 TMA producer, 9 MMAs
// (leader), 10 statistics of the query tiles (keys kernel).
//
// The queries kernel is launched first and the keys kernel as its programmatic
// dependent: the keys kernel's CTAs take SMs as the queries kernel's leave, which they
// need not wait for (its CTAs have all passed their own wait for the pass over the
// outputs by then), only before their own end.  Items are handed out to whichever
// pair is free.
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
constexpr int kThreads = 32 * 11;
constexpr int kScoreWarps = 8, kProducerWarp = 8, kMmaWarp = 9, kStatWarp = 10;
constexpr int kTile = 128;   // rows of a tile
constexpr int kBlock = 256;  // rows of an item
constexpr int kStatSlots = 2;
constexpr int kItemSlots = 4;

template <int D, bool kKeys>
struct Smem {
  static constexpr uint32_t kOwn = 128 * D * 2;    // this CTA's 128 rows of one operand
  static constexpr uint32_t kHalf = 64 * D * 2;    // half a tile's rows, or its columns of all rows
  static constexpr int kNStages = kKeys ? 2 : 3, kDStages = 2;
  static constexpr uint32_t kNBytes = 2 * kHalf, kDBytes = (kKeys ? 2 : 1) * kHalf;  // one CTA's bytes of a stage
  static constexpr uint32_t kN = 2 * kOwn;                      // rows ring
  static constexpr uint32_t kD = kN + kNStages * kNBytes;       // columns ring
  static constexpr uint32_t kStage = kD + kDStages * kDBytes;   // epilogue: 32 rows x 64 columns per warp
  static constexpr uint32_t kStat = kStage + kScoreWarps * 4096;
  static constexpr uint32_t kBars = kStat + (kKeys ? kStatSlots * 1024 : 0);
  static constexpr int kOwnFull = 0, kOwnEmpty = 1, kNFull = 2, kNEmpty = kNFull + kNStages, kDFull = kNEmpty + kNStages,
                       kDEmpty = kDFull + kDStages, kSDone = kDEmpty + kDStages, kPDone = kSDone + 1, kSUsed = kPDone + 2,
                       kDsFull = kSUsed + 1, kAccDone = kDsFull + 2, kAccFree = kAccDone + 1, kStatFull = kAccFree + 1,
                       kStatEmpty = kStatFull + kStatSlots, kItemFull = kStatEmpty + kStatSlots,
                       kItemEmpty = kItemFull + kItemSlots, kMmaDone = kItemEmpty + kItemSlots, kNumBars = kMmaDone + 1;
  // warps that read each item from the ring: the leader's MMA warp, the follower's
  // producer, and the score (and statistics) warps of both
  static constexpr int kItemTakers = 2 + 2 * kScoreWarps + (kKeys ? 2 : 0);
  static constexpr uint32_t kTmemHolder = kBars + 8 * kNumBars;
  static constexpr uint32_t kAbort = kTmemHolder + 4, kPeerAbort = kAbort + 4;
  static constexpr uint32_t kLoadRec = kPeerAbort + 4;  // each CTA's loads: own rows, rows ring, columns ring
  static constexpr uint32_t kItemRing = kLoadRec + 24;
  static constexpr uint32_t kUsed = kItemRing + 4 * kItemSlots;
  static constexpr uint32_t kMaxDynamic = 232448;
  static constexpr uint32_t kDynamic = kUsed + 1024 < kMaxDynamic ? kUsed + 1024 : kMaxDynamic;
  static_assert(kUsed <= kMaxDynamic, "shared-memory layout too large");
};

// The MMAs of one product.  Offsets are in 16-byte units of a descriptor.
// Rows by rows (over the head dim): A is this CTA's 128 rows, B 64 rows, both in
// boxes of 64 columns.
template <int D>
__device__ __forceinline__ void mma_rows(uint32_t d_tmem, uint64_t a, uint64_t b) {
  constexpr uint32_t kIdesc = idesc_bf16_f32(256, kTile, false);
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk)
    tc2_mma_ss(d_tmem, a + (((kk >> 2) * 16384u + (kk & 3) * 32u) >> 4), b + (((kk >> 2) * 8192u + (kk & 3) * 32u) >> 4), kIdesc,
               kk > 0 ? 1u : 0u);
}
// Weights (128 of them a row, bf16 in tensor memory, the second 64 at +64 columns)
// by a tile's columns.
template <int D>
__device__ __forceinline__ void mma_cols(uint32_t d_tmem, uint32_t w_tmem, uint64_t b, uint32_t accumulate) {
  constexpr uint32_t kIdesc = idesc_bf16_f32(256, D, true);
#pragma unroll
  for (int kk = 0; kk < kTile / 16; ++kk)
    tc2_mma_ts(d_tmem, w_tmem + static_cast<uint32_t>((kk >> 2) * 64 + (kk & 3) * 8), b + ((16u * D * kk) >> 4), kIdesc,
               kk > 0 ? 1u : accumulate);
}
template <int D>
__device__ __forceinline__ uint64_t cols_desc(uint32_t addr) {
  return D == 64 ? sdesc_sw64(addr, 128 * D, 512) : sdesc_sw128(addr, 128 * D, 1024);
}

// 64 columns of this thread's lane, and their bf16 pairs back over the first 32.
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

// One warp's 32 rows x 64 columns (chunks [chunk0, chunk0 + 8) of 16 bytes of each
// row) through shared memory, so that whole 128-byte lines are written.
struct RowsOut {
  uint32_t stage;  // this warp's 4 KB
  int lane;
  __device__ __forceinline__ void put(int chunk, uint4 v) const {
    st_shared_v4(stage + 128u * lane + (static_cast<uint32_t>(chunk ^ (lane & 7)) << 4), v);
  }
  // rows [0, rows) of the warp go to dst + row * stride
  __device__ __forceinline__ void flush(__nv_bfloat16* dst, int64_t stride, int rows) const {
    __syncwarp();
    const int r0 = lane >> 3, ch = lane & 7;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = 4 * i + r0;
      const uint4 v = ld_shared_v4(stage + 128u * r + (static_cast<uint32_t>(ch ^ (r & 7)) << 4));
      if (r < rows) *reinterpret_cast<uint4*>(dst + r * stride + 8 * ch) = v;
    }
    __syncwarp();
  }
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
  // Items reach the warps through a ring in the shared memory of both CTAs.  The
  // leader's producer (one lane) passes on item k, -1 when none is left:
  __device__ __forceinline__ bool publish(int k, int item) const {
    const int s = k % kItemSlots;
    if (k >= kItemSlots && !(wait(L::kItemEmpty + s, k / kItemSlots - 1, 81) &&
                             mbar_try_wait_acquire_cluster(bar(L::kItemEmpty + s), static_cast<uint32_t>(k / kItemSlots - 1) & 1u)))
      return false;
    const uint32_t at = base + L::kItemRing + 4u * static_cast<uint32_t>(s);
    st_cluster_u32(mapa_shared(at, 0), static_cast<uint32_t>(item));
    st_cluster_u32(mapa_shared(at, 1), static_cast<uint32_t>(item));
    mbar_arrive_release_cluster(mapa_shared(bar(L::kItemFull + s), 0));
    mbar_arrive_release_cluster(mapa_shared(bar(L::kItemFull + s), 1));
    return true;
  }
  // and the other roles take it, a whole warp (`lanes` 32) or one lane alone; -2: gave up.
  __device__ __forceinline__ int take(int k, bool whole_warp) const {
    const int s = k % kItemSlots;
    const uint32_t parity = static_cast<uint32_t>(k / kItemSlots) & 1u;
    bool ok = wait(L::kItemFull + s, k / kItemSlots, 82) && mbar_try_wait_acquire_cluster(bar(L::kItemFull + s), parity);
    if (whole_warp) ok = __all_sync(0xffffffffu, ok);
    if (!ok) return -2;
    const int item = *reinterpret_cast<const volatile int*>(ptr + L::kItemRing + 4 * s);
    if (whole_warp) __syncwarp();
    if (!whole_warp || lane == 0) mbar_arrive_release_cluster(lbar(L::kItemEmpty + s));
    return whole_warp ? __shfl_sync(0xffffffffu, item, 0) : item;
  }
};
// The leader's choice of items: its cluster's index first, then the next of the
// list (a counter that the pass over the outputs has set to zero), or every
// n_clusters-th without a counter.
struct Chooser {
  int* work;
  int cluster, n_clusters, n_items;
  int k = 0;  // items chosen
  __device__ __forceinline__ int next() {
    const int64_t it = k == 0 ? cluster : work ? static_cast<int64_t>(n_clusters) + atomicAdd(work, 1)
                                               : cluster + static_cast<int64_t>(k) * n_clusters;
    ++k;
    return it < n_items ? static_cast<int>(it) : -1;
  }
};

// Returns false where the block has to leave (both CTAs of the pair alike).  late:
// the wait for the kernel before this one is at the end (BwdArgs::behind_queries).
template <typename L>
__device__ __forceinline__ bool enter(Cta<L>& c, uint8_t* smem, const BwdArgs& a, const BwdMaps& maps, bool late) {
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
      const bool scores = i == L::kSUsed || i == L::kDsFull || i == L::kDsFull + 1 || i == L::kAccFree;
      const bool local = i >= L::kStatEmpty && i < L::kStatEmpty + kStatSlots;
      const bool items = i >= L::kItemEmpty && i < L::kItemEmpty + kItemSlots;
      mbar_init(c.bar(i), scores ? 2 * kScoreWarps : local ? kScoreWarps : items ? L::kItemTakers : 1);
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
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  c.ctl = Ctl{abort_flag, a.timeout_ns, a.status};
  if (!late) grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
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

// Teardown, after the roles (the producer's counts are in `own`, `rows`, `cols` of
// its lane 0).  As in attn_tc2_kernel: when neither CTA gave up, every load was
// waited for by the MMAs that read it; else the leader arms or counts what the
// other CTA's half lacks, and waits for the last phase of each barrier.
template <typename L>
__device__ __forceinline__ void leave(const Cta<L>& c, int own, int rows, int cols) {
  if (c.warp == kProducerWarp && c.lane == 0) {
    const uint32_t rec = mapa_shared(c.base + L::kLoadRec + 12u * c.rank, 0);
    st_cluster_u32(rec, static_cast<uint32_t>(own));
    st_cluster_u32(rec + 4, static_cast<uint32_t>(rows));
    st_cluster_u32(rec + 8, static_cast<uint32_t>(cols));
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
    auto settle = [&](int b, int n, int slots, int slot, uint32_t bytes) {
      auto loads = [&](uint32_t total) { return (static_cast<int>(total) - slot + slots - 1) / slots; };
      int m = loads(mine[n]);
      const int theirs = loads(mine[3 + n]);
      if (theirs == m + 1) {
        mbar_arrive_expect_tx(c.bar(b), bytes);
        m = theirs;
      } else if (m == theirs + 1) {
        mbar_complete_tx(c.bar(b), bytes);
      }
      if (m > 0) tc::drain_one(c.bar(b), static_cast<uint32_t>(m - 1) & 1u, c.ctl.timeout_ns);
    };
    settle(L::kOwnFull, 0, 1, 0, 2 * L::kOwn);
#pragma unroll 1
    for (int s = 0; s < L::kNStages; ++s) settle(L::kNFull + s, 1, L::kNStages, s, L::kNBytes);
#pragma unroll 1
    for (int s = 0; s < L::kDStages; ++s) settle(L::kDFull + s, 2, L::kDStages, s, L::kDBytes);
  }
  cluster_sync();
}
}  // namespace bwd

template <int D>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(bwd::kThreads, 1)
    attn_bwd_keys_kernel(const __grid_constant__ BwdMaps maps, const __grid_constant__ BwdKeys keys, const __grid_constant__ BwdArgs args) {
  using namespace bwd;
  using L = Smem<D, true>;
  constexpr uint32_t kColS = 0, kColP = 128, kColV = 256, kColK = 384;
  extern __shared__ uint8_t smem_raw[];
  Cta<L> c;
  if (!enter(c, smem_raw, args, maps, args.behind_queries != 0)) return;
  const int cluster = static_cast<int>(blockIdx.x >> 1), n_clusters = static_cast<int>(gridDim.x >> 1);
  const int n_items = keys.n_tiles * args.num_heads;
  struct Item {
    int head, row0, rows, q0, q_rows, nt, in_b, add_from, add_row0;
  };
  auto item_of = [&](int it) -> Item {
    Item t;
    const BwdItem i = bwd_item(keys, it, args.num_heads);
    t.head = i.head;
    const BwdKeySeg& s = keys.seg[i.seg];
    const int r0 = i.tile * kBlock;
    t.row0 = s.k_row0 + r0;
    t.rows = min(kBlock, s.k_rows - r0);
    t.q0 = s.q_row0;
    t.q_rows = s.q_rows;
    t.nt = (s.q_rows + kTile - 1) / kTile;
    t.in_b = s.in_b;
    t.add_from = s.add_from - r0;  // within the item
    t.add_row0 = s.add_row0 + r0;
    return t;
  };
  int own = 0, nn = 0, nd = 0;  // loads issued
  if (c.warp == kProducerWarp) {
    if (c.lane == 0) {
      Chooser choose{args.work_keys, cluster, n_clusters, n_items};
      int it = c.leader ? choose.next() : 0;
      if (c.leader && !c.publish(0, it)) it = -2;
#pragma unroll 1
      for (int k = 0;; ++k) {
        if (!c.leader) it = c.take(k, false);
        if (it < 0) break;
        int ahead = c.leader ? choose.next() : 0;  // used two tiles later
        const Item t = item_of(it);
        if (t.nt == 0) {
          if (c.leader && !c.publish(k + 1, ahead)) break;
          it = ahead;
          continue;
        }
        const int x = t.head * D, xc = x + D / 2 * static_cast<int>(c.rank);
        if (own > 0 && !c.wait(L::kOwnEmpty, own - 1, 31)) break;
        if (c.leader) mbar_arrive_expect_tx(c.bar(L::kOwnFull), 4 * L::kOwn);
        const int y = t.row0 + 128 * static_cast<int>(c.rank);
        load_own<D>(c.base, t.in_b ? &maps.kb : &maps.ka, c.lbar(L::kOwnFull), x, y);
        load_own<D>(c.base + L::kOwn, t.in_b ? &maps.vb : &maps.va, c.lbar(L::kOwnFull), x, y);
        ++own;
        bool ok = true;
#pragma unroll 1
        for (int j = 0; j < t.nt; ++j) {
          const int y0 = t.q0 + kTile * j;
          const int ns = nn % L::kNStages, ds = nd % L::kDStages;
          if (nn >= L::kNStages && !(ok = c.wait(L::kNEmpty + ns, nn / L::kNStages - 1, 32))) break;
          if (c.leader) mbar_arrive_expect_tx(c.bar(L::kNFull + ns), 2 * L::kNBytes);
          const uint32_t n = c.base + L::kN + ns * L::kNBytes;
          load_half<D>(n, &maps.q, c.lbar(L::kNFull + ns), x, y0 + 64 * static_cast<int>(c.rank));
          load_half<D>(n + L::kHalf, &maps.d_o, c.lbar(L::kNFull + ns), x, y0 + 64 * static_cast<int>(c.rank));
          ++nn;
          if (nd >= L::kDStages && !(ok = c.wait(L::kDEmpty + ds, nd / L::kDStages - 1, 33))) break;
          if (c.leader) mbar_arrive_expect_tx(c.bar(L::kDFull + ds), 2 * L::kDBytes);
          const uint32_t d = c.base + L::kD + ds * L::kDBytes;
          tma_load_2d_pair(d, &maps.cols0, c.lbar(L::kDFull + ds), xc, y0);
          tma_load_2d_pair(d + L::kHalf, &maps.cols1, c.lbar(L::kDFull + ds), xc, y0);
          ++nd;
          if (c.leader && j == min(1, t.nt - 1) && !(ok = c.publish(k + 1, ahead))) break;
        }
        if (!ok) break;
        it = ahead;
      }
    }
    __syncwarp();
  } else if (c.warp == kMmaWarp) {
    if (c.leader) {
      const uint64_t kd = sdesc_sw128(c.base, 16, 1024), vd = sdesc_sw128(c.base + L::kOwn, 16, 1024);
      const uint64_t nd0 = sdesc_sw128(c.base + L::kN, 16, 1024), dd0 = cols_desc<D>(c.base + L::kD);
      const uint32_t tm = c.tmem;
      bool issued = false;
      int t = 0, k = 0;  // tiles, and items with tiles, so far
#pragma unroll 1
      for (int i = 0;; ++i) {
        const int it = c.take(i, true);
        if (it < 0) break;
        const int nt = __shfl_sync(0xffffffffu, item_of(it).nt, 0);
        if (nt == 0) continue;
        // S and dP of tile i (dP's commit also frees the tile's rows)
        auto slot = [&](int i) { return nd0 + static_cast<uint64_t>(i % L::kNStages) * (L::kNBytes >> 4); };
        auto cols = [&](int i) { return dd0 + static_cast<uint64_t>(i % L::kDStages) * (L::kDBytes >> 4); };
        auto issue_s = [&](int i) {
          mma_rows<D>(tm + kColS, kd, slot(i));
          tc2_commit_mc(c.bar(L::kSDone), 3);
        };
        auto issue_dp = [&](int i, bool last) {
          mma_rows<D>(tm + kColP, vd, slot(i) + (L::kHalf >> 4));
          tc2_commit_mc(c.bar(L::kPDone), 3);
          tc2_commit_mc(c.bar(L::kNEmpty + i % L::kNStages), 3);
          if (last) tc2_commit_mc(c.bar(L::kOwnEmpty), 3);
        };
        if (!c.wait_all(L::kOwnFull, k, 34) || !c.wait_all(L::kNFull + t % L::kNStages, t / L::kNStages, 35)) goto mma_done;
        issued = true;
        if (elect_one()) {
          tc_fence_after();
          issue_s(t);
          issue_dp(t, nt == 1);
        }
        __syncwarp();
#pragma unroll 1
        for (int j = 0; j < nt; ++j, ++t) {
          const bool next = j + 1 < nt;
          if (!c.wait_all(L::kDFull + t % L::kDStages, t / L::kDStages, 36)) goto mma_done;
          if (j == 0 && k > 0 && !c.wait_all(L::kAccFree, k - 1, 37)) goto mma_done;
          if (next && !c.wait_all(L::kNFull + (t + 1) % L::kNStages, (t + 1) / L::kNStages, 35)) goto mma_done;
          if (!c.wait_all(L::kSUsed, t, 38)) goto mma_done;  // P is written
          if (elect_one()) {
            tc_fence_after();
            mma_cols<D>(tm + kColV, tm + kColS, cols(t), j > 0 ? 1u : 0u);
            if (next) issue_s(t + 1);
          }
          __syncwarp();
          if (!c.wait_all(L::kDsFull, t, 39)) goto mma_done;
          if (elect_one()) {
            tc_fence_after();
            mma_cols<D>(tm + kColK, tm + kColP, cols(t) + (L::kHalf >> 4), j > 0 ? 1u : 0u);
            tc2_commit_mc(c.bar(L::kDEmpty + t % L::kDStages), 3);
            if (next)
              issue_dp(t + 1, j + 2 == nt);
            else
              tc2_commit_mc(c.bar(L::kAccDone), 3);
          }
          __syncwarp();
        }
        ++k;
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
    for (int i = 0; ok; ++i) {
      const int it = c.take(i, true);
      if (it < 0) break;
      const Item m = item_of(it);
      const float2* src = args.stats + m.head * args.rows + m.q0;
#pragma unroll 1
      for (int j = 0; j < m.nt; ++j, ++t) {
        float2 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = kTile * j + 32 * i + c.lane;
          v[i] = r < m.q_rows ? src[r] : make_float2(INFINITY, 0.f);
        }
        const int s = t % kStatSlots;
        if (t >= kStatSlots && !(ok = c.wait_all(L::kStatEmpty + s, t / kStatSlots - 1, 40))) break;
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
    const uint32_t lanes = static_cast<uint32_t>(lane0) << 16;
    const uint32_t t_s = c.tmem + lanes + kColS + 64 * half, t_p = c.tmem + lanes + kColP + 64 * half;
    const f32x2 sl2 = make_f32x2(args.scale_log2, args.scale_log2);
    const uint32_t l_used = c.lbar(L::kSUsed), l_ds = c.lbar(L::kDsFull), l_free = c.lbar(L::kAccFree);
    auto arrive = [&](uint32_t b) {
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (c.lane == 0) mbar_arrive_cluster(b);
    };
    int t = 0, k = 0;
#pragma unroll 1
    for (int i = 0;; ++i) {
      const int it = c.take(i, true);
      if (it < 0) break;
      const Item m = item_of(it);
#pragma unroll 1
      for (int j = 0; j < m.nt; ++j, ++t) {
        const int s = t % kStatSlots;
        const uint32_t stat = c.base + L::kStat + 1024u * s + 256u * half;
        float p[64];
        if (!c.wait_all(L::kStatFull + s, t / kStatSlots, 41) || !c.wait_all(L::kSDone, t, 42)) goto scores_done;
        tc_fence_after();
        load64(t_s, p);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t pk[16];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const float4 nl = ld_shared_f4(stat + 128u * h + 16u * q);
            float* x = p + 32 * h + 4 * q;
            float e0, e1, e2, e3;
            split_f32x2(fma_f32x2(make_f32x2(x[0], x[1]), sl2, make_f32x2(nl.x, nl.y)), e0, e1);
            split_f32x2(fma_f32x2(make_f32x2(x[2], x[3]), sl2, make_f32x2(nl.z, nl.w)), e2, e3);
            x[0] = ex2_approx(e0), x[1] = ex2_approx(e1), x[2] = ex2_approx(e2), x[3] = ex2_approx(e3);
            pk[2 * q] = pack_bf16x2(x[0], x[1]);
            pk[2 * q + 1] = pack_bf16x2(x[2], x[3]);
          }
          tmem_st16(t_s + 16u * h, pk);
        }
        arrive(l_used);
        if (!c.wait_all(L::kPDone, t, 43)) goto scores_done;
        tc_fence_after();
        {
          float d[64];
          load64(t_p, d);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t pk[16];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const float4 ndl = ld_shared_f4(stat + 512u + 128u * h + 16u * q);
              const int i = 32 * h + 4 * q;
              float e0, e1, e2, e3;
              split_f32x2(mul_f32x2(make_f32x2(p[i], p[i + 1]), add_f32x2(make_f32x2(d[i], d[i + 1]), make_f32x2(ndl.x, ndl.y))), e0, e1);
              split_f32x2(mul_f32x2(make_f32x2(p[i + 2], p[i + 3]), add_f32x2(make_f32x2(d[i + 2], d[i + 3]), make_f32x2(ndl.z, ndl.w))), e2,
                          e3);
              pk[2 * q] = pack_bf16x2(e0, e1);
              pk[2 * q + 1] = pack_bf16x2(e2, e3);
            }
            tmem_st16(t_p + 16u * h, pk);
          }
        }
        arrive(l_ds);
        if (c.lane == 0) mbar_arrive(c.bar(L::kStatEmpty + s));
      }
      // dV (warps 0-3) and dK (warps 4-7) of this warp's 32 keys
      if (m.nt > 0) {
        if (!c.wait_all(L::kAccDone, k, 44)) goto scores_done;
        tc_fence_after();
        ++k;
      }
      const int row = 128 * static_cast<int>(c.rank) + lane0;  // the warp's first row in the item
      const float scale = half ? args.scale : 1.f;
      __nv_bfloat16* out = half ? (m.in_b ? args.dkb : args.dka) : (m.in_b ? args.dvb : args.dva);
      const __nv_bfloat16* add = half ? args.add_k : args.add_v;
      const bool adds = row + c.lane >= m.add_from && row + c.lane < m.rows;
      const __nv_bfloat16* from = adds ? add + (static_cast<int64_t>(m.add_row0) + row + c.lane) * args.row_stride + m.head * D : nullptr;
      out += (static_cast<int64_t>(m.row0) + row) * args.row_stride + m.head * D;
      const RowsOut rows{c.base + L::kStage + 4096u * c.warp, c.lane};
#pragma unroll
      for (int cc = 0; cc < D / 64; ++cc) {
        float v[64];
        if (m.nt > 0) {
          load64(c.tmem + lanes + (half ? kColK : kColV) + 64 * cc, v);
        } else {
#pragma unroll
          for (int i = 0; i < 64; ++i) v[i] = 0.f;
        }
        if (cc + 1 == D / 64 && m.nt > 0) {  // all of it is read
          tc_fence_before();
          __syncwarp();
          if (c.lane == 0) mbar_arrive_cluster(l_free);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          Vec8 x;
#pragma unroll
          for (int e = 0; e < 8; ++e) x.v[e] = v[8 * q + e] * scale;
          if (adds) {
            const Vec8 y = unpack8(*reinterpret_cast<const uint4*>(from + 64 * cc + 8 * q));
#pragma unroll
            for (int e = 0; e < 8; ++e) x.v[e] += y.v[e];
          }
          rows.put(q, pack8(x));
        }
        rows.flush(out + 64 * cc, args.row_stride, m.rows - row);
      }
    }
  scores_done:;
  }
  leave(c, own, nn, nd);
  if (args.behind_queries) grid_dependency_wait();  // the work after this kernel sees both
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
  if (!enter(c, smem_raw, args, maps, false)) return;
  const int cluster = static_cast<int>(blockIdx.x >> 1), n_clusters = static_cast<int>(gridDim.x >> 1);
  const int n_items = queries.n_tiles * args.num_heads;
  struct Item {
    int head, row0, rows, a0, a_len, b0, b_len, na, nt;
  };
  auto item_of = [&](int it) -> Item {
    Item t;
    const BwdItem i = bwd_item(queries, it, args.num_heads);
    t.head = i.head;
    const BwdQuerySeg& s = queries.seg[i.seg];
    const int r0 = i.tile * kBlock;
    t.row0 = s.q_row0 + r0;
    t.rows = min(kBlock, s.q_rows - r0);
    t.a0 = s.a_row0, t.a_len = s.a_len, t.b0 = s.b_row0, t.b_len = s.b_len;
    t.na = (s.a_len + kTile - 1) / kTile;
    t.nt = t.na + (s.b_len + kTile - 1) / kTile;
    return t;
  };
  int own = 0, nn = 0, nd = 0;  // loads issued
  if (c.warp == kProducerWarp) {
    if (c.lane == 0) {
      Chooser choose{args.work_queries, cluster, n_clusters, n_items};
      int it = c.leader ? choose.next() : 0;
      if (c.leader && !c.publish(0, it)) it = -2;
#pragma unroll 1
      for (int k = 0;; ++k) {
        if (!c.leader) it = c.take(k, false);
        if (it < 0) break;
        int ahead = c.leader ? choose.next() : 0;  // used two tiles later
        const Item t = item_of(it);
        const int x = t.head * D, xc = x + D / 2 * static_cast<int>(c.rank);
        if (own > 0 && !c.wait(L::kOwnEmpty, own - 1, 51)) break;
        if (c.leader) mbar_arrive_expect_tx(c.bar(L::kOwnFull), 4 * L::kOwn);
        const int y = t.row0 + 128 * static_cast<int>(c.rank);
        load_own<D>(c.base, &maps.q, c.lbar(L::kOwnFull), x, y);
        load_own<D>(c.base + L::kOwn, &maps.d_o, c.lbar(L::kOwnFull), x, y);
        ++own;
        bool ok = true;
#pragma unroll 1
        for (int j = 0; j < t.nt; ++j) {
          const bool b = j >= t.na;
          const int y0 = b ? t.b0 + kTile * (j - t.na) : t.a0 + kTile * j;
          const int ns = nn % L::kNStages, ds = nd % L::kDStages;
          if (nn >= L::kNStages && !(ok = c.wait(L::kNEmpty + ns, nn / L::kNStages - 1, 52))) break;
          if (c.leader) mbar_arrive_expect_tx(c.bar(L::kNFull + ns), 2 * L::kNBytes);
          const uint32_t n = c.base + L::kN + ns * L::kNBytes;
          load_half<D>(n, b ? &maps.kb : &maps.ka, c.lbar(L::kNFull + ns), x, y0 + 64 * static_cast<int>(c.rank));
          load_half<D>(n + L::kHalf, b ? &maps.vb : &maps.va, c.lbar(L::kNFull + ns), x, y0 + 64 * static_cast<int>(c.rank));
          ++nn;
          if (nd >= L::kDStages && !(ok = c.wait(L::kDEmpty + ds, nd / L::kDStages - 1, 53))) break;
          if (c.leader) mbar_arrive_expect_tx(c.bar(L::kDFull + ds), 2 * L::kDBytes);
          tma_load_2d_pair(c.base + L::kD + ds * L::kDBytes, b ? &maps.cols1 : &maps.cols0, c.lbar(L::kDFull + ds), xc, y0);
          ++nd;
          if (c.leader && j == min(1, t.nt - 1) && !(ok = c.publish(k + 1, ahead))) break;
        }
        if (!ok) break;
        it = ahead;
      }
    }
    __syncwarp();
  } else if (c.warp == kMmaWarp) {
    if (c.leader) {
      const uint64_t qd = sdesc_sw128(c.base, 16, 1024), od = sdesc_sw128(c.base + L::kOwn, 16, 1024);
      const uint64_t nd0 = sdesc_sw128(c.base + L::kN, 16, 1024), dd0 = cols_desc<D>(c.base + L::kD);
      const uint32_t tm = c.tmem;
      bool issued = false;
      int t = 0;
#pragma unroll 1
      for (int k = 0;; ++k) {
        const int it = c.take(k, true);
        if (it < 0) break;
        const int nt = __shfl_sync(0xffffffffu, item_of(it).nt, 0);
        if (!c.wait_all(L::kOwnFull, k, 54)) goto mma_done;
        // step j: S and dP of tile j, then dQ of tile j - 1
#pragma unroll 1
        for (int j = 0; j <= nt; ++j) {
          if (j < nt) {
            const int i = t + j, s = i % L::kNStages;
            if (!c.wait_all(L::kNFull + s, i / L::kNStages, 55)) goto mma_done;
            if (i > 0 && !c.wait_all(L::kSUsed, i - 1, 56)) goto mma_done;
            issued = true;
            if (elect_one()) {
              tc_fence_after();
              const uint64_t b = nd0 + static_cast<uint64_t>(s) * (L::kNBytes >> 4);
              mma_rows<D>(tm + kColS, qd, b);
              tc2_commit_mc(c.bar(L::kSDone), 3);
              mma_rows<D>(tm + kColP + 128u * (i & 1), od, b + (L::kHalf >> 4));
              tc2_commit_mc(c.bar(L::kPDone + (i & 1)), 3);
              tc2_commit_mc(c.bar(L::kNEmpty + s), 3);
              if (j + 1 == nt) tc2_commit_mc(c.bar(L::kOwnEmpty), 3);
            }
            __syncwarp();
          }
          if (j > 0) {
            const int i = t + j - 1, s = i % L::kDStages;
            if (!c.wait_all(L::kDFull + s, i / L::kDStages, 57)) goto mma_done;
            if (j == 1 && k > 0 && !c.wait_all(L::kAccFree, k - 1, 58)) goto mma_done;
            if (!c.wait_all(L::kDsFull + (i & 1), i >> 1, 59)) goto mma_done;
            if (elect_one()) {
              tc_fence_after();
              mma_cols<D>(tm + kColQ, tm + kColP + 128u * (i & 1), dd0 + static_cast<uint64_t>(s) * (L::kDBytes >> 4), j > 1 ? 1u : 0u);
              tc2_commit_mc(c.bar(L::kDEmpty + s), 3);
              if (j == nt) tc2_commit_mc(c.bar(L::kAccDone), 3);
            }
            __syncwarp();
          }
        }
        t += nt;
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
    int t = 0;
#pragma unroll 1
    for (int k = 0;; ++k) {
      const int it = c.take(k, true);
      if (it < 0) break;
      const Item m = item_of(it);
      const int row = 128 * static_cast<int>(c.rank) + lane0;  // the warp's first row in the item
      const float2 st = row + c.lane < m.rows ? args.stats[m.head * args.rows + m.row0 + row + c.lane] : make_float2(INFINITY, 0.f);
      const f32x2 nl = make_f32x2(-st.x, -st.x), ndl = make_f32x2(-st.y, -st.y);
#pragma unroll 1
      for (int j = 0; j < m.nt; ++j, ++t) {
        float p[64];
        if (!c.wait_all(L::kSDone, t, 61)) goto scores_done;
        tc_fence_after();
        const int valid = (j < m.na ? m.a_len - kTile * j : m.b_len - kTile * (j - m.na)) - 64 * half;  // of this warp's 64 keys
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
        const int b = t & 1;
        if (!c.wait_all(L::kPDone + b, t >> 1, 62)) goto scores_done;
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
      // dQ: columns [D / 2 half, D / 2 (half + 1)) of this warp's 32 rows
      if (!c.wait_all(L::kAccDone, k, 63)) goto scores_done;
      tc_fence_after();
      {
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
        // staged as chunks of 16 bytes: 8 a row, or 4 of each of the two warps at D = 64
        const RowsOut rows{c.base + L::kStage + 4096u * c.warp, c.lane};
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
      }
    }
  scores_done:;
  }
  leave(c, own, nn, nd);
}

}  // namespace rc
