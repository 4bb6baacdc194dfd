// f8_wgrad.cuh -- a weight's gradient, dw = add + dy^T x, from bf16 dy [rows, n] and x [rows, k]
// in its 8-bit form: bf16 tcgen05 MMAs over CTA pairs, 256 columns of x times 256 (or 128) of
// dy a tile.
//
// The sum runs over the rows, along which x has a scale each, so the tensor core cannot
// apply them.  A code times its power of two is exact in bf16 (from 2^-126 on, and 2^128 is taken as the largest value): a first kernel writes x's
// values, or a panel of their columns, to the workspace, and the product is that of dy and of the
// values that x stands for.  (Turned into bf16 on the way to the MMAs, a code is converted once for
// each 256 columns of dy: eight warps took 766 cycles for what 512 cycles of MMAs
// need, 435 us for 4608 rows and 16384 x 4096, where the first kernel takes 10.)
//
// CTA r of a pair holds columns [128 r, 128 r + 128) of x's tile and half of dy's; both
// lie as they come, columns contiguous (MN-major).  A stage is 64 rows, 32 KB, 512 cycles of
// MMAs.  Sums: two buffers of 256 columns of tensor memory, lane = column of x, so that each
// store of a lane joins those of its warp in one line of dw.  The tensor core cuts off
// what does not fit when it adds, so that an error grows with the rows (1.7e-6 of dw's norm at
// 4608); each 1024 rows' sums are therefore added up, rounded to nearest, in the registers of
// eight warps (4e-7), which write a tile while the MMAs of the next one run.  Where the tiles
// are few the rows are split and the parts added by another kernel in a fixed order.
//
// What bounds it: a stage's loads, 592 cycles for 512 of MMAs (588 with half of the MMAs left out: the loads alone; 529 with half of the
// loads; 444 with half of both: each side has a part that does not shrink with its work), and the power cap.  4608 rows, 16384 x 4096: 350
// to 391 us on different GPUs, 1.58 to 1.77 PFLOP/s (0.84 to 0.93 of measured).
#pragma once
#include "f8_pair.cuh"
#include "vec8.cuh"

namespace rc {
namespace f8 {

struct WgradArgs {
  const void* add;      // like dw, or null
  void* dw;             // [n, k], ld elements between rows; the parts, fp32 [n, k] each, where there are several
  int64_t ld;
  int32_t f32;          // dw (and add) fp32, else bf16
  int32_t n, k, bn;     // k: columns of this panel; bn: columns of dy in a tile, 128 or 256
  int32_t stages;       // of 64 rows
  int32_t splits, per_split;  // parts, and stages of each
  Tiles tiles;                // m: of n; n: of k
  int32_t n_whole, n_items;   // tiles taken whole (of all parts); these and the halves, of 128 columns of dy, of the others
  Guard guard;
};
struct WgradMaps {
  CUtensorMap dy, x;  // 64 rows x 64 columns (128 bytes)
};

struct WgradSmem {
  static constexpr int kSlots = 6, kSlots2 = 0;
  static constexpr int kChunk = 16;  // stages whose sums are taken out together
  static constexpr uint32_t kOperand = 16384, kSlot = 2 * kOperand, kBars = kSlots * kSlot;
  static constexpr int kFull = 0, kFull2 = 0, kEmpty = kFull + kSlots, kAccFull = kEmpty + kSlots, kAccEmpty = kAccFull + 2, kDone = kAccEmpty + 2,
                       kNumBars = kDone + 1;
  static constexpr uint32_t kAux = kBars + 8 * kNumBars, kUsed = kAux + kAuxBytes, kDynamic = kUsed + 1024;
  static constexpr int kProducer = 8, kMma = 9, kProducer2 = 10, kThreads = 32 * 11;  // warps 0-7: sums; 8: loads of x; 10: of dy
  static_assert(kDynamic <= kMaxDynamic, "shared-memory layout too large");
  __device__ static constexpr uint32_t arrivals(int i) { return i >= kAccEmpty && i < kDone ? 16 : 1; }  // eight warps of each CTA
};

// The items of a launch: part by part, each over all tiles; without parts, the tiles behind the last full round over the
// pairs in halves where these are no more than the pairs (a stage of one takes 384 cycles, of a tile 512: 1500 rows,
// 4112 x 2064, 153 tiles: 33.6 -> 32.4 us; 4608 rows, 16384 x 4096, 1024 tiles: 362 -> 356).
struct WgradItem {
  int row0, bn, j, part, first, last;  // rows of dw, columns in 256s, stages [first, last)
};
__device__ __forceinline__ WgradItem wgrad_item(const WgradArgs& a, int item) {
  const int n_tiles = a.tiles.m * a.tiles.n, half = item - a.n_whole;
  const int tile = half < 0 ? item : a.n_whole + (half >> 1);
  WgradItem t;
  int i;
  t.part = tile / n_tiles;
  a.tiles.at(tile - t.part * n_tiles, &i, &t.j);
  t.bn = half < 0 ? a.bn : 128;
  t.row0 = i * a.bn + (half < 0 ? 0 : 128 * (half & 1));
  t.first = t.part * a.per_split;
  t.last = min(a.stages, t.first + a.per_split);
  return t;
}

// What comes before the product: x's values and d_bias, by blocks of one kernel.  Bound by memory, and in small calls
// by the launches (two kernels: 333 rows, x of 272 and dy of 1040 columns, 17.3 us a call from the host, one 14.0; 4608 rows, x of 4096 and
// dy of 16384: 406 and 399).
constexpr int kInputBlocks = 8;  // of a cluster
constexpr int kInputThreads = 256;

// Two values in bf16; above its largest, that (NaNs as they are).
__device__ __forceinline__ uint32_t pack_finite_bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Columns [col0, col0 + cols) of rows in 8-bit form as bf16 [rows, cols]: 16 columns a thread.
__device__ __forceinline__ void write_values(const Rows& r, int col0, int cols, uint16_t* to, int block, int blocks) {
  const int strips = cols / 16;
  const int64_t n = r.rows * strips, step = static_cast<int64_t>(blocks) * kInputThreads;
  for (int64_t i = static_cast<int64_t>(block) * kInputThreads + threadIdx.x; i < n; i += step) {
    const int64_t row = i / strips;
    const int col = static_cast<int>(i - row * strips) * 16;
    const uint4 c = *reinterpret_cast<const uint4*>(r.codes + row * r.width + col0 + col);
    const float s = from_codes(r.scales[row * r.pitch + (col0 + col) / kBlock]);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    uint32_t out[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 v = unpack_e4m3x4(w[j]);
      out[2 * j] = pack_finite_bf16x2(v.x * s, v.y * s), out[2 * j + 1] = pack_finite_bf16x2(v.z * s, v.w * s);
    }
    uint4* y = reinterpret_cast<uint4*>(to + row * cols + col);
    y[0] = make_uint4(out[0], out[1], out[2], out[3]);
    y[1] = make_uint4(out[4], out[5], out[6], out[7]);
  }
}

// d_bias: the sums of dy over the rows.  A cluster of kInputBlocks blocks has 64 columns, eight a thread; each
// block takes every kInputBlocks-th 32 rows, and the first one adds up what the others found, in their order.
__device__ __forceinline__ void write_bias_grad(const uint16_t* dy, int64_t ld, int64_t rows, int n, float* out, int col0) {
  __shared__ __align__(16) float part[32][64];
  __shared__ __align__(16) float all[kInputBlocks][64];
  cluster_sync();  // (the others' shared memory is there)
  const int lane = threadIdx.x & 7, sub = threadIdx.x >> 3;
  const int col = col0 + 8 * lane, rank = static_cast<int>(cluster_ctarank());
  Vec8 v = fill8(0.f);
  if (col < n) {
#pragma unroll 4
    for (int64_t r = 32 * rank + sub; r < rows; r += 32 * kInputBlocks) {
      const Vec8 x = unpack8(*reinterpret_cast<const uint4*>(dy + r * ld + col));
#pragma unroll
      for (int e = 0; e < 8; ++e) v.v[e] += x.v[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) part[sub][8 * lane + e] = v.v[e];
  __syncthreads();
  if (threadIdx.x < 64) {
    float s = 0.f;
    for (int i = 0; i < 32; ++i) s += part[i][threadIdx.x];
    st_cluster_u32(mapa_shared(smem_u32(&all[rank][threadIdx.x]), 0), __float_as_uint(s));
  }
  cluster_sync();
  if (rank == 0 && threadIdx.x < 64 && col0 + static_cast<int>(threadIdx.x) < n) {
    float s = 0.f;
    for (int i = 0; i < kInputBlocks; ++i) s += all[i][threadIdx.x];
    out[col0 + threadIdx.x] = s;
  }
}
// The first `bias_clusters` clusters have d_bias.
__global__ void __cluster_dims__(kInputBlocks, 1, 1) __launch_bounds__(kInputThreads)
    f8_wgrad_inputs_kernel(const Rows r, int col0, int cols, uint16_t* values, const uint16_t* dy, int64_t ld, int n, float* d_bias, int bias_clusters) {
  grid_dependency_wait();
  grid_launch_dependents();
  const int block = static_cast<int>(blockIdx.x) - bias_clusters * kInputBlocks;
  if (block < 0)
    write_bias_grad(dy, ld, r.rows, n, d_bias, static_cast<int>(blockIdx.x / kInputBlocks) * 64);
  else
    write_values(r, col0, cols, values, block, static_cast<int>(gridDim.x) - bias_clusters * kInputBlocks);
}

// One lane's column of x, up to 128 rows of dw (the first `rows` of them there), each a line's part with the
// other lanes'.  What is added comes first, then the sums, then all is stored.
// (The pointers go from row to row: with the rows' addresses kept for the whole tile the registers spill.)
template <typename T>
__device__ __forceinline__ void next_row(T& p, int64_t stride) {
  p += stride;
  asm volatile("" : "+l"(p));
}
template <typename T>
__device__ __forceinline__ void load_rows(float (&v)[128], const T* from, int64_t stride, int rows) {
#pragma unroll
  for (int e = 0; e < 128; ++e) {
    v[e] = 0.f;
    if (e < rows) v[e] = sizeof(T) == 4 ? __uint_as_float(static_cast<uint32_t>(*from)) : __uint_as_float(static_cast<uint32_t>(*from) << 16);
    next_row(from, stride);
  }
}
template <typename T>
__device__ __forceinline__ void store_rows(const float (&v)[128], T* to, int64_t stride, int rows) {
#pragma unroll
  for (int e = 0; e < 128; ++e) {
    if (e < rows) *to = sizeof(T) == 4 ? static_cast<T>(__float_as_uint(v[e])) : static_cast<T>(pack_bf16x2(v[e], 0.f));
    next_row(to, stride);
  }
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(WgradSmem::kThreads, 1)
    f8_wgrad_kernel(const __grid_constant__ WgradMaps maps, const __grid_constant__ WgradArgs a) {
  using L = WgradSmem;
  extern __shared__ uint8_t smem_raw[];
  Cta<L> c;
  if (!c.enter(smem_raw, a.guard)) return;
  const int cluster = static_cast<int>(blockIdx.x >> 1), n_clusters = static_cast<int>(gridDim.x >> 1);
  const int n_items = a.n_items;
  auto bytes = [](int bn) { return make_uint2(L::kOperand, static_cast<uint32_t>(bn) * 64u); };  // of one CTA's load: x, dy
  int loads = 0;
  if (c.warp == L::kProducer || c.warp == L::kProducer2) {
    if (c.lane == 0) {
      const bool of_x = c.warp == L::kProducer, arms = of_x && c.leader;
      const int most = of_x ? loads_before_stop(a.guard.stop, c.rank) : 0x7FFFFFFF;
      const CUtensorMap* map = of_x ? &maps.x : &maps.dy;
      const uint32_t to = c.base + (of_x ? 0u : L::kOperand);
      bool ok = true;
#pragma unroll 1
      for (int item = cluster; ok && item < n_items; item += n_clusters) {
        const WgradItem t = wgrad_item(a, item);
        // (the maps count bytes)
        const int x = 2 * (of_x ? t.j * 256 + 128 * static_cast<int>(c.rank) : t.row0 + t.bn / 2 * static_cast<int>(c.rank));
        const bool two = of_x || t.bn > 128;  // 64 columns a load
        const uint2 b = bytes(t.bn);
#pragma unroll 1
        for (int st = t.first; st < t.last; ++st) {
          const int s = loads % L::kSlots, n = loads / L::kSlots;
          ok = loads != most && (n == 0 || c.wait(L::kEmpty + s, n - 1, 111));
          if (!ok) break;
          const uint32_t at = to + static_cast<uint32_t>(s) * L::kSlot, full = c.lbar(L::kFull + s);
          if (arms) mbar_arrive_expect_tx(c.bar(L::kFull + s), 2 * (b.x + b.y));
          tma_load_2d_pair(at, map, full, x, st * 64);
          if (two) tma_load_2d_pair(at + 8192, map, full, x + 128, st * 64);
          ++loads;
        }
      }
    }
    __syncwarp();
  } else if (c.warp == L::kMma) {
    if (c.leader) {
      // (64 columns of 64 rows are 8 KB; 8 rows 1 KB)
      const uint64_t ad = sdesc_sw128(c.base, 8192, 1024), bd = sdesc_sw128(c.base + L::kOperand, 8192, 1024);
      bool issued = false, ok = true;
      int load = 0, used = 0;  // stages, chunks
#pragma unroll 1
      for (int item = cluster; ok && item < n_items; item += n_clusters) {
        const WgradItem t = wgrad_item(a, item);
        const uint32_t idesc = idesc_bf16_f32(256, t.bn, true) | (1u << 15);  // A MN-major too
#pragma unroll 1
        for (int st = t.first, in_chunk = 0; st < t.last; ++st, ++load) {
          const int s = load % L::kSlots;
          ok = (in_chunk > 0 || used < 2 || c.wait_all(L::kAccEmpty + (used & 1), (used >> 1) - 1, 113)) && c.wait_all(L::kFull + s, load / L::kSlots, 114);
          if (!ok) break;
          issued = true;
          const bool end = in_chunk + 1 == L::kChunk || st + 1 == t.last;
          if (elect_one()) {
            tc_fence_after();
            const uint32_t d = c.tmem + 256u * (used & 1);
            const uint64_t off = static_cast<uint64_t>(s) * (L::kSlot >> 4);
#pragma unroll
            for (int q = 0; q < 4; ++q) tc2_mma_ss(d, ad + off + 128 * q, bd + off + 128 * q, idesc, in_chunk > 0 || q > 0 ? 1u : 0u);
            tc2_commit_mc(c.bar(L::kEmpty + s), 3);
            if (end) tc2_commit_mc(c.bar(L::kAccFull + (used & 1)), 3);
          }
          __syncwarp();
          in_chunk = end ? 0 : in_chunk + 1;
          used += end ? 1 : 0;
        }
      }
      c.finish_mmas(issued);
    }
  } else {
    // A warp has half of dw's rows, 128 (or 64) of them, of 32 columns of x.
    const int group = c.warp >> 2, quarter = c.warp & 3;
    int used = 0;
    bool ok = true;
#pragma unroll 1
    for (int item = cluster; ok && item < n_items; item += n_clusters) {
      const WgradItem t = wgrad_item(a, item);
      const int col = t.j * 256 + 128 * static_cast<int>(c.rank) + 32 * quarter + c.lane;
      const int half = t.bn / 2, row0 = t.row0 + half * group, rows = col < a.k ? min(half, a.n - row0) : 0;
      const int64_t ld = a.splits == 1 ? a.ld : a.k, at = (static_cast<int64_t>(t.part) * (a.splits == 1 ? 0 : a.n) + row0) * ld + col;
      float v[128];  // (what is to be added first: it is on its way while the MMAs run)
      if (a.add == nullptr || a.splits > 1) {
#pragma unroll
        for (int e = 0; e < 128; ++e) v[e] = 0.f;
      } else if (a.f32) {
        load_rows(v, static_cast<const uint32_t*>(a.add) + at, ld, rows);
      } else {
        load_rows(v, static_cast<const uint16_t*>(a.add) + at, ld, rows);
      }
#pragma unroll 1
      for (int st = t.first; ok && st < t.last; st += L::kChunk, ++used) {
        ok = c.wait_all(L::kAccFull + (used & 1), used >> 1, 120);
        if (!ok) break;
        tc_fence_after();
        const uint32_t from = c.tmem + 256u * (used & 1) + static_cast<uint32_t>(half * group) + (static_cast<uint32_t>(quarter) << 21);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          if (16 * q >= half) break;
          uint32_t r[16];
          tmem_ld16(from + 16 * q, r);
          tmem_wait_ld(r);
#pragma unroll
          for (int e = 0; e < 16; ++e) v[16 * q + e] += __uint_as_float(r[e]);
        }
        tc_fence_before();
        __syncwarp();
        if (c.lane == 0) mbar_arrive_cluster(c.lbar(L::kAccEmpty + (used & 1)));
      }
      if (!ok) break;
      if (a.f32)
        store_rows(v, static_cast<uint32_t*>(a.dw) + at, ld, rows);
      else
        store_rows(v, static_cast<uint16_t*>(a.dw) + at, ld, rows);
    }
  }
  const int whole = cluster < a.n_whole ? (a.n_whole - cluster + n_clusters - 1) / n_clusters : 0;  // tiles of this pair
  c.leave(Loads{loads, bytes(a.bn), bytes(a.n_whole < n_items ? 128 : a.bn), whole * a.stages}, Loads{});
}

// dw = add + the parts, one after the other.
__global__ void __launch_bounds__(256) f8_wgrad_sum_kernel(const float* parts, int n_parts, int64_t n, const void* add, void* dw, int f32) {
  grid_dependency_wait();
  grid_launch_dependents();
  const int64_t step = static_cast<int64_t>(gridDim.x) * 256 * 8;
  for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8; i < n; i += step) {
    Vec8 v = fill8(0.f);
    for (int p = 0; p < n_parts; ++p) {
      const Vec8 x = load_param8(parts, p * n + i, true);
#pragma unroll
      for (int e = 0; e < 8; ++e) v.v[e] += x.v[e];
    }
    if (add) {
      const Vec8 x = load_param8(add, i, f32 != 0);
#pragma unroll
      for (int e = 0; e < 8; ++e) v.v[e] += x.v[e];
    }
    if (f32) {
      float4* y = reinterpret_cast<float4*>(static_cast<float*>(dw) + i);
      y[0] = make_float4(v.v[0], v.v[1], v.v[2], v.v[3]);
      y[1] = make_float4(v.v[4], v.v[5], v.v[6], v.v[7]);
    } else {
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(dw) + i) = pack8(v);
    }
  }
}

}  // namespace f8
}  // namespace rc
