// f8_few.cuh -- f8_linear's products where the rows are too few for tiles of 256: the
// weight is streamed once, 128 of its rows (columns of y) as the first operand of
// block-scaled MMAs (M = 128), up to 128 rows of x as the second (N = rows, a multiple of 16).
//
// What bounds it is the weight's bytes: 2 rows, 24576 x 4096: 21.5 us a call, 4.7 TB/s (0.69 of the measured copy; a launch and its
// first loads are 6 of it).  Two CTAs an SM, each with up to 100 KB of loads in
// flight, cover the memory's latency; where 128-row tiles alone would leave SMs idle, a
// cluster of up to eight CTAs splits x's columns, and each of them adds up every so-manieth
// row of y from the others' shared memory, in their order, with a warp to a row: one block of 128
// columns, so that GELU and the 8-bit form need nothing else.
#pragma once
#include "f8_linear.cuh"

namespace rc {
namespace f8 {

struct FewArgs {
  Out o;
  int32_t x_chunks, w_chunks;  // of 128 rows
  int32_t k;                   // columns of x
  int32_t per;                 // blocks of 128 of them for each CTA of a cluster, a multiple of 4
  int32_t n, slots;            // rows of a tile as the MMAs take them, a multiple of 16; stages that fit
  Guard guard;
};

struct FewSmem {
  static constexpr int kMaxSlots = 6, kScaleSlots = 4;
  static constexpr uint32_t kStages = 104 * 1024, kA = 16384, kScales = kStages, kBars = kScales + kScaleSlots * 1024;
  static constexpr int kFull = 0, kEmpty = kFull + kMaxSlots, kScFull = kEmpty + kMaxSlots, kScEmpty = kScFull + kScaleSlots, kAccFull = kScEmpty + kScaleSlots,
                       kAccEmpty = kAccFull + 1, kNumBars = kAccEmpty + 1;
  static constexpr uint32_t kAux = kBars + 8 * kNumBars, kUsed = kAux + 8, kDynamic = kUsed + 1024;
  static constexpr int kProducer = 4, kMma = 5, kThreads = 32 * 6;  // warps 0-3: sums
  static constexpr uint32_t kTmemCols = 256, kTmemScales = 128;      // 8 columns a slot
  static_assert(kDynamic <= 113 * 1024, "two CTAs an SM");
  __host__ __device__ static constexpr uint32_t slot_bytes(int n) { return kA + 128u * n; }
  static constexpr int rows_of_tile(int64_t rows) { return rows < 128 ? (static_cast<int>(rows) + 15) / 16 * 16 : 128; }
};

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void* tmap, uint32_t bar, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void mx_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

// Grid: (CTAs of a cluster, tiles of 128 columns of y, tiles of 128 rows).  kLong: a CTA has more than kSumBlocks blocks of
// columns, after each of which the sums go into registers (f8_linear.cuh).
template <int kEpi, bool kLong>
__global__ void __launch_bounds__(FewSmem::kThreads, 2)
    f8_few_kernel(const __grid_constant__ LinearMaps maps, const __grid_constant__ FewArgs a) {
  using L = FewSmem;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  volatile int* aux = reinterpret_cast<volatile int*>(smem_raw + (base - raw) + L::kAux);
  const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int split = static_cast<int>(blockIdx.x), row0 = static_cast<int>(blockIdx.z) * 128, col0 = static_cast<int>(blockIdx.y) * 128;
  const int rows = static_cast<int>(min(static_cast<int64_t>(128), a.o.rows - row0)), n = a.n;
  const int blocks = (a.k + kBlock - 1) / kBlock, first = split * a.per, last = min(blocks, first + a.per);
  const uint32_t slot_bytes = L::slot_bytes(n);
  auto bar = [&](int i) { return base + L::kBars + 8u * static_cast<uint32_t>(i); };
  auto wait = [&](int i, int k, int where) {
    const uint32_t parity = static_cast<uint32_t>(k) & 1u;
    return mbar_try_wait(bar(i), parity) || wait_more(bar(i), parity, aux, a.guard.status, a.guard.timeout_ns, where);
  };
  auto wait_all = [&](int i, int k, int where) { return __all_sync(0xffffffffu, wait(i, k, where)); };
  if (threadIdx.x == 0) {
    for (int i = 0; i < L::kNumBars; ++i) mbar_init(bar(i), i == L::kAccEmpty ? 4 : 1);
    aux[0] = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == L::kMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + L::kAux + 4), "r"(L::kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, static_cast<uint32_t>(aux[1]), 0);
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();

  // CTAs begin in different places of their columns: all at the same one, they would ask the same
  // memory channels for rows that lie a power of two apart
  const int begin = first + 4 * (static_cast<int>(blockIdx.y * 5) % ((last - first + 3) / 4));
  auto next = [&](int kb) { return kb + 1 == last ? first : kb + 1; };
  int loads = 0, groups = 0;
  if (warp == L::kProducer) {
    if (lane == 0) {
      const int most = loads_before_stop(a.guard.stop, static_cast<uint32_t>(split & 1));
      bool ok = true;
#pragma unroll 1
      for (int i = first, kb = begin; i < last; ++i, kb = next(kb)) {
        if ((kb & 3) == 0) {
          const int s = groups % L::kScaleSlots, k = groups / L::kScaleSlots;
          ok = k == 0 || wait(L::kScEmpty + s, k - 1, 132);
          if (!ok) break;
          const uint32_t at = base + L::kScales + 1024u * s;
          mbar_arrive_expect_tx(bar(L::kScFull + s), 1024);
          tma_load_2d(at, &maps.w_tiles, bar(L::kScFull + s), 0, (kb >> 2) * a.w_chunks + col0 / 128);
          tma_load_2d(at + 512, &maps.x_tiles, bar(L::kScFull + s), 0, (kb >> 2) * a.x_chunks + row0 / 128);
          ++groups;
        }
        const int s = loads % a.slots, k = loads / a.slots;
        ok = loads != most && (k == 0 || wait(L::kEmpty + s, k - 1, 131));
        if (!ok) break;
        const uint32_t at = base + static_cast<uint32_t>(s) * slot_bytes;
        mbar_arrive_expect_tx(bar(L::kFull + s), slot_bytes);
        tma_load_2d(at, &maps.w, bar(L::kFull + s), kb * kBlock, col0);
        tma_load_2d(at + L::kA, &maps.x, bar(L::kFull + s), kb * kBlock, row0);
        ++loads;
      }
    }
    __syncwarp();
  } else if (warp == L::kMma) {
    const uint64_t sd = scales_desc(base + L::kScales);
    const uint32_t idesc = idesc_mx(128, n);
    int load = 0, group = 0, sums = 0;  // sums: committed
    bool ok = true, issued = false;     // issued: since the last of these
#pragma unroll 1
    for (int i = first, kb = begin; i < last; ++i, ++load) {
      const int s = load % a.slots, sc = group % L::kScaleSlots, in_sum = kLong ? load % kSumBlocks : load;
      const uint32_t sfa = tmem + L::kTmemScales + 8u * sc;
      ok = (!kLong || in_sum > 0 || sums == 0 || wait_all(L::kAccEmpty, sums - 1, 133)) &&
           ((kb & 3) != 0 || wait_all(L::kScFull + sc, group / L::kScaleSlots, 134)) && wait_all(L::kFull + s, load / a.slots, 135);
      if (!ok) break;
      issued = true;
      const int steps = min(4, (a.k - kb * kBlock + 31) / 32);
      const bool end = i + 1 == last, out = end || (kLong && in_sum == kSumBlocks - 1);
      const int after = next(kb);
      if (elect_one()) {
        tc_fence_after();
        if ((kb & 3) == 0) {
          const uint64_t at = sd + static_cast<uint64_t>(sc) * (1024 >> 4);
          copy_scales(sfa, at);
          copy_scales(sfa + 4, at + (512 >> 4));
        }
        const uint32_t at = base + static_cast<uint32_t>(s) * slot_bytes;
        const uint64_t ad = sdesc_sw128(at, 16, 1024), bd = sdesc_sw128(at + L::kA, 16, 1024);
        const uint32_t id = idesc_byte(idesc, kb & 3);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q < steps) mx_mma(tmem, ad + 2 * q, bd + 2 * q, id, sfa, sfa + 4, in_sum > 0 || q > 0 ? 1u : 0u);
        commit(bar(L::kEmpty + s));
        if ((after & 3) == 0 || end) commit(bar(L::kScEmpty + sc));
        if (out) commit(bar(L::kAccFull));
      }
      __syncwarp();
      if ((after & 3) == 0 || end) ++group;
      if (out) ++sums, issued = false;
      kb = after;
    }
    // (always: the sums' warps may have given up on MMAs that go on)
    if (elect_one()) {
      if (issued) commit(bar(L::kAccFull));
      if (issued || sums > 0) drain(bar(L::kAccFull), static_cast<uint32_t>(issued ? sums : sums - 1) & 1u, a.guard.timeout_ns);
    }
    __syncwarp();
  } else {
    // The sums as [row][128 columns of y] into the stages' memory: every load has been read.
    const uint32_t to = base + 4u * (32 * warp + lane);
    if (kLong) {
      const int sums = (last - first + kSumBlocks - 1) / kSumBlocks;
      float v[128];
#pragma unroll
      for (int e = 0; e < 128; ++e) v[e] = 0.f;
      int i = 0;
#pragma unroll 1
      for (; i < sums; ++i) {
        if (!wait_all(L::kAccFull, i, 136)) break;
        tc_fence_after();
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          if (16 * q >= n) break;
          uint32_t r[16];
          tmem_ld16(tmem + 16 * q + (static_cast<uint32_t>(warp) << 21), r);
          tmem_wait_ld(r);
#pragma unroll
          for (int e = 0; e < 16; ++e) v[16 * q + e] += __uint_as_float(r[e]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(L::kAccEmpty));
      }
      if (i == sums) {
#pragma unroll
        for (int e = 0; e < 128; ++e)
          if (e < n) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + 512u * e), "r"(__float_as_uint(v[e])) : "memory");
      }
    } else if (wait_all(L::kAccFull, 0, 136)) {
      tc_fence_after();
#pragma unroll 1
      for (int r = 0; r < n; r += 16) {
        uint32_t v[16];
        tmem_ld16(tmem + r + (static_cast<uint32_t>(warp) << 21), v);
        tmem_wait_ld(v);
#pragma unroll
        for (int e = 0; e < 16; ++e) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + 512u * (r + e)), "r"(v[e]) : "memory");
      }
    }
  }
  tc_fence_before();
  cluster_sync();
  if (aux[0] && warp == L::kProducer && lane == 0) {  // a wait ran out: loads may still be on their way
    for (int s = 0; s < a.slots; ++s)
      if (loads > s) drain(bar(L::kFull + s), static_cast<uint32_t>((loads - s - 1) / a.slots) & 1u, a.guard.timeout_ns);
    for (int s = 0; s < L::kScaleSlots; ++s)
      if (groups > s) drain(bar(L::kScFull + s), static_cast<uint32_t>((groups - s - 1) / L::kScaleSlots) & 1u, a.guard.timeout_ns);
  }
  if (warp == L::kMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L::kTmemCols) : "memory");
  }
  const int splits = static_cast<int>(gridDim.x);
  if (warp < 4) {
#pragma unroll 1
    for (int r = split + splits * warp; r < rows; r += 4 * splits) {
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
      for (int s = 0; s < splits; ++s) {
        const float4 x = ld_cluster_f4(mapa_shared(base + 512u * r + 16u * lane, s));
        v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
      }
      finish_row<kEpi>(a.o, row0 + r, col0, lane, v);
    }
  }
  cluster_sync();  // (the others may still read this CTA's sums)
}

}  // namespace f8
}  // namespace rc
