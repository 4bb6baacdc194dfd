// f8_pair.cuh -- what the 8-bit products' kernels share: bounded waits, the set-up and
// teardown of a CTA pair (a cluster of two, cta_group::2 MMAs with M = 256), the
// block-scaled MMA, and the order in which tiles are taken.
//
// Every wait is bounded; one that runs out sets the device's error word and the CTA's
// abort flag, on which every role leaves its loop.  Before tensor memory is freed and
// the CTA exits, the MMAs issued and the loads in flight are waited for (again bounded).
#pragma once
#include <cuda.h>

#include "f8_common.cuh"

namespace rc {
namespace f8 {

constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kMaxDynamic = 232448;
constexpr int kTimeoutBase = 0x1000;  // of the error word: refcache_status subtracts it

struct Guard {  // of a launch
  int* status;  // the device's error word
  uint64_t timeout_ns;
  int32_t stop;  // fault injection: load before which a producer stops, bit 9: of the second CTA
};

struct Ctl {
  volatile int* abort_flag;
  int* status;
  uint64_t timeout_ns;
};

// (not a function of its own: ptxas allots no registers beside a call where warpgroups change theirs)
__device__ __forceinline__ bool wait_more(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status, uint64_t timeout_ns, int where) {
  const uint64_t t0 = globaltimer_ns();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 16; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    if (globaltimer_ns() - t0 > timeout_ns) {
      *abort_flag = 1;
      atomicCAS(status, 0, kTimeoutBase + where);
      return false;
    }
  }
}
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity, uint64_t timeout_ns) {
  const uint64_t t0 = globaltimer_ns();
  while (!mbar_try_wait(bar, parity))
    if (globaltimer_ns() - t0 > timeout_ns) break;
}

// ---------------------------------------------------------------- block-scaled MMAs
// kind::mxf8f6f4: instruction descriptor bits 4-5 which byte of B's scale words, 7-9 and
// 10-12 the operands' formats (0: E4M3), 17-22 N >> 3, 23 scales are UE8M0, 27-28 M >> 7,
// 29-30 which byte of A's scale words.  An MMA takes 32 codes of each row; with one
// scale for 128, four MMAs in a row name the same byte and a word serves 512 columns.
__host__ __device__ constexpr uint32_t idesc_mx(int m, int n) {
  return (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) | (static_cast<uint32_t>(m >> 7) << 27);
}
__device__ __forceinline__ uint32_t idesc_byte(uint32_t idesc, uint32_t byte) { return idesc | byte << 4 | byte << 29; }
__device__ __forceinline__ void mx_mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(acc)
      : "memory");
}
// 128 rows' scale words (Rows::tiles) from shared memory into four columns of tensor memory:
// row r into lane r % 32 of each 32 lanes, column r / 32.
__device__ __forceinline__ uint64_t scales_desc(uint32_t addr) {  // no swizzle, 8 rows of 16 bytes each 128 bytes
  return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(128 >> 4) << 32) | (1ull << 46);
}
__device__ __forceinline__ void copy_scales_pair(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}

// Registers of a warpgroup, all four warps alike: fewer than at launch, or more, of what others gave
// up.  On a path of its own for each: after a join the compiler would count with the fewest.
template <int kRegs>
__device__ __forceinline__ void fewer_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs));
}
template <int kRegs>
__device__ __forceinline__ void more_registers() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs));
}

// ---------------------------------------------------------------- a CTA of a pair
// L: kNumBars, kBars, kAux (abort flag, tensor memory's address, the other CTA's abort
// flag, the loads of both CTAs' producers), kUsed, kDynamic, arrivals(barrier), kDone, the warps
// kProducer, kProducer2 and kMma, and two rings of loads: their first barriers kFull and kFull2, kSlots
// and kSlots2.  Both producers of both CTAs load into each slot of a ring (getting one load out takes a
// thread 150 cycles, so that one producer alone was busy for 390 of the 512 cycles that a stage's MMAs
// run); the first CTA's first one arms the barrier, on which all of them complete.
constexpr uint32_t kAuxBytes = 12 + 4 * 8;
struct Loads {
  int n;                     // issued
  uint2 bytes, bytes_last;   // of one, by the first producer and by the second; of the last tile's loads
  int before_last;           // loads before these
};
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
    const uint32_t parity = static_cast<uint32_t>(n) & 1u;
    return mbar_try_wait(bar(i), parity) || wait_more(bar(i), parity, ctl.abort_flag, ctl.status, ctl.timeout_ns, where);
  }
  __device__ __forceinline__ bool wait_all(int i, int n, int where) const { return __all_sync(0xffffffffu, wait(i, n, where)); }

  // Returns false (in both CTAs alike) where the block has to leave at once.
  __device__ __forceinline__ bool enter(uint8_t* smem, const Guard& g) {
    const uint32_t raw = smem_u32(smem);
    base = (raw + 1023u) & ~1023u;
    ptr = smem + (base - raw);
    rank = cluster_ctarank();
    leader = rank == 0;
    warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    lane = threadIdx.x & 31;
    if (base - raw + L::kUsed > L::kDynamic) {
      grid_dependency_wait();
      if (threadIdx.x == 0) atomicCAS(g.status, 0, kTimeoutBase + 198);
      return false;
    }
    volatile int* aux = reinterpret_cast<volatile int*>(ptr + L::kAux);
    if (threadIdx.x == 0) {
      for (int i = 0; i < L::kNumBars; ++i) mbar_init(bar(i), L::arrivals(i));
      aux[0] = 0;
      fence_barrier_init();
      fence_proxy_async_smem();
    }
    if (warp == L::kMma) {
      tmem_alloc_pair(base + L::kAux + 4, kTmemCols);
      tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    ctl = Ctl{aux, g.status, g.timeout_ns};
    tmem = __shfl_sync(0xffffffffu, static_cast<uint32_t>(aux[1]), 0);
    grid_dependency_wait();
    if (threadIdx.x == 0) grid_launch_dependents();
    return true;
  }

  // The MMA warp's last act: what it issued is done.
  __device__ __forceinline__ void finish_mmas(bool issued) const {
    __syncwarp();
    if (issued && elect_one()) {
      tc2_commit_mc(bar(L::kDone), 1);
      drain(bar(L::kDone), 0u, ctl.timeout_ns);
    }
    __syncwarp();
  }

  // Of each ring, what a producer (lane 0 of both) loaded.  When neither CTA gave up, every load was waited for by the MMAs that read it; else
  // the leader arms or counts what some of the four lack of the others and waits for the last phase of each slot.
  __device__ __forceinline__ void leave(const Loads& loads, const Loads& loads2) const {
    if ((warp == L::kProducer || warp == L::kProducer2) && lane == 0) {
      const uint32_t at = mapa_shared(base + L::kAux + 12 + 16 * rank + (warp == L::kProducer ? 0 : 8), 0);
      st_cluster_u32(at, static_cast<uint32_t>(loads.n));
      st_cluster_u32(at + 4, static_cast<uint32_t>(loads2.n));
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0) st_cluster_u32(mapa_shared(base + L::kAux + 8, rank ^ 1u), static_cast<uint32_t>(*ctl.abort_flag));
    cluster_sync();
    if (warp == L::kMma) {
      tc_fence_after();
      tmem_dealloc_pair(tmem, kTmemCols);
    }
    const volatile int* aux = reinterpret_cast<const volatile int*>(ptr + L::kAux);
    if (aux[0] == 0 && aux[2] == 0) return;
    if (leader && warp == L::kProducer && lane == 0) {
      auto settle = [&](int full, int slots, int ring, const Loads& of) {
#pragma unroll 1
        for (int slot = 0; slot < slots; ++slot) {
          int most = 0, n[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {  // the arming one first
            n[i] = (aux[3 + 2 * i + ring] - slot + slots - 1) / slots;
            most = max(most, n[i]);
          }
          const uint2 b = slot + (most - 1) * slots < of.before_last ? of.bytes : of.bytes_last;
          uint32_t there = 0, lacking = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) (n[i] == most ? there : lacking) += i & 1 ? b.y : b.x;
          if (n[0] < most)
            mbar_arrive_expect_tx(bar(full + slot), there);
          else if (lacking)
            mbar_complete_tx(bar(full + slot), lacking);
          if (most > 0) drain(bar(full + slot), static_cast<uint32_t>(most - 1) & 1u, ctl.timeout_ns);
        }
      };
      settle(L::kFull, L::kSlots, 0, loads);
      settle(L::kFull2, L::kSlots2, 1, loads2);
    }
    cluster_sync();
  }
};

// Loads until a producer stops: all of them, but for fault injection.
__device__ __forceinline__ int loads_before_stop(int stop, uint32_t rank) {
  return stop != 0 && static_cast<uint32_t>((stop >> 9) & 1) == rank ? (stop & 255) - 1 : 0x7FFFFFFF;
}

// Tile t of a grid of m x n: bands of eight rows of tiles, so that the tiles that run at
// one time share rows and columns in the L2.
struct Tiles {
  int32_t m, n;
  __device__ __forceinline__ void at(int t, int* i, int* j) const {
    const int band = t / (8 * n), r = t - band * 8 * n, rows = min(8, m - band * 8);
    *j = r / rows;
    *i = band * 8 + r - *j * rows;
  }
};

}  // namespace f8
}  // namespace rc
