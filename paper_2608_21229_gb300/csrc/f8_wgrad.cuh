// f8_wgrad.cuh -- a weight's gradient, dw = add + dy^T x, from bf16 dy [rows, n] and x [rows, k]
// in its 8-bit form: bf16 tcgen05 MMAs over CTA pairs, 256 x 256 (or 128) of dw a tile.
//
// The sum runs over the rows, along which x has a scale each, so the tensor core cannot
// apply them.  A code times its power of two is exact in bf16: eight warps of each CTA turn 64
// rows of codes into bf16 in the shared memory that the MMAs read, and the product is that of
// dy and of the values that x stands for.  Both operands lie with the rows of dw and its
// columns contiguous (MN-major), as they come.
//
// CTA r of a pair holds columns [128 r, 128 r + 128) of dy's tile and half of x's.  A stage
// is 64 rows: 16 KB of dy by TMA, 8 KB of codes (and 512 bytes of scales) by TMA into a
// ring of their own, 16 KB of bf16, in which the MMAs take 512 cycles.  The converted
// operand of the second CTA is read by MMAs that the first one issues: its warps arrive
// at a barrier of their own CTA, and a warp passes that on with release at cluster scope
// to one of the first CTA that acquires it and opens the MMA warp's barrier; either takes
// longer than a stage has (about 1000 cycles), so two warps of each CTA take turns.
//
// Sums: two buffers of 256 columns of tensor memory; four warps write one out while the
// other is added to.  Where the tiles are few the rows are split and the parts added by
// another kernel in a fixed order.
#pragma once
#include "f8_pair.cuh"

namespace rc {
namespace f8 {

struct WgradArgs {
  const void* add;   // [n, k] like dw, or null
  void* dw;          // [n, k]; the parts, fp32, where there are several
  int32_t f32;       // dw (and add) fp32, else bf16
  int32_t n, k, bn;  // bn: columns of a tile, 128 or 256
  int64_t rows;
  int32_t chunks;  // of 128 rows
  int32_t stages;  // of 64 rows
  int32_t splits, per_split;  // parts, and stages of each
  Tiles tiles;
  Guard guard;
};
struct WgradMaps {
  CUtensorMap dy, codes, tiles;  // 64 rows x 64 columns (128 bytes); 64 rows x half a tile's columns; 512 bytes
};

struct WgradSmem {
  static constexpr int kSlots = 4, kSlots2 = 6, kSlotsB = 6;  // dy, codes, converted
  static constexpr bool kOwn2 = true;  // codes complete on barriers of the CTA that loads them
  static constexpr int kAhead = 3;                            // stages that codes are loaded ahead of dy
  static constexpr uint32_t kA = 16384, kCodes = 8192, kC = kCodes + 512, kB = 16384;
  static constexpr uint32_t kOffA = 0, kOffB = kSlots * kA, kOffC = kOffB + kSlotsB * kB, kBars = kOffC + kSlots2 * kC;
  // kFull2 and kEmpty2 are of each CTA's own codes; kBDone: converted, in this CTA; kBPeer: in the other one; kBFull: in both
  static constexpr int kFull = 0, kEmpty = kFull + kSlots, kFull2 = kEmpty + kSlots, kEmpty2 = kFull2 + kSlots2, kBDone = kEmpty2 + kSlots2,
                       kBPeer = kBDone + kSlotsB, kBFull = kBPeer + kSlotsB, kBEmpty = kBFull + kSlotsB, kAccFull = kBEmpty + kSlotsB,
                       kAccEmpty = kAccFull + 2, kDone = kAccEmpty + 2, kNumBars = kDone + 1;
  static constexpr uint32_t kAux = kBars + 8 * kNumBars, kUsed = kAux + 28, kDynamic = kUsed + 1024;
  // warps 0-3: sums, 4-11: codes into bf16
  static constexpr int kConvert = 4, kConvertWarps = 8, kProducer = 12, kMma = 13, kRelay = 14, kThreads = 32 * 16;
  static_assert(kDynamic <= kMaxDynamic, "shared-memory layout too large");
  __device__ static constexpr uint32_t arrivals(int i) {
    return (i >= kEmpty2 && i < kBPeer) || (i >= kAccEmpty && i < kDone) ? 8 : 1;  // kEmpty2, kBDone: the converting warps; kAccEmpty: four warps of each CTA
  }
};

// Four codes times s (a power of two in both halves, or NaN) as four bf16.  A code's bits
// shifted to bf16's places are its value times 2^-120, E4M3's subnormals being bf16's.
__device__ __forceinline__ uint2 codes_to_bf16(uint32_t c, uint32_t s) {
  auto two = [&](uint32_t h) {  // codes in the upper bytes
    const uint32_t v = ((h >> 4) & 0x07F007F0u) | (h & 0x80008000u);
    __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&v);
    const uint32_t up = 0x7B807B80u;  // 2^120
    x = __hmul2(__hmul2(x, *reinterpret_cast<const __nv_bfloat162*>(&up)), *reinterpret_cast<const __nv_bfloat162*>(&s));
    return *reinterpret_cast<const uint32_t*>(&x);
  };
  return make_uint2(two(__byte_perm(c, 0, 0x1404)), two(__byte_perm(c, 0, 0x3424)));
}

__host__ __device__ constexpr uint32_t idesc_wgrad(int n) { return idesc_bf16_f32(256, n, true) | (1u << 15); }

// The items of a launch: part by part, each over all tiles.
struct WgradItem {
  int i, j, part, first, last;  // stages [first, last)
};
__device__ __forceinline__ WgradItem wgrad_item(const WgradArgs& a, int item) {
  const int n_tiles = a.tiles.m * a.tiles.n;
  WgradItem t;
  t.part = item / n_tiles;
  a.tiles.at(item - t.part * n_tiles, &t.i, &t.j);
  t.first = t.part * a.per_split;
  t.last = min(a.stages, t.first + a.per_split);
  return t;
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(WgradSmem::kThreads, 1)
    f8_wgrad_kernel(const __grid_constant__ WgradMaps maps, const __grid_constant__ WgradArgs a) {
  using L = WgradSmem;
  extern __shared__ uint8_t smem_raw[];
  Cta<L> c;
  if (!c.enter(smem_raw, a.guard)) return;
  const int cluster = static_cast<int>(blockIdx.x >> 1), n_clusters = static_cast<int>(gridDim.x >> 1);
  const int n_items = a.tiles.m * a.tiles.n * a.splits, half = a.bn / 2;  // half: columns of x in a CTA
  const uint32_t code_bytes = static_cast<uint32_t>(half) * 64u, c_bytes = code_bytes + 512u;
  int loads = 0, loads2 = 0;
  if (c.warp == L::kProducer) {
    if (c.lane == 0) {
      const int most = loads_before_stop(a.guard.stop, c.rank);
      // codes go kAhead stages ahead of dy: they are needed earlier by their conversion
      int item2 = cluster, at2 = -1;
      WgradItem t2{};
      auto next_codes = [&]() -> bool {  // false: gave up
        if (at2 < 0) {
          if (item2 >= n_items) return true;
          t2 = wgrad_item(a, item2);
          at2 = t2.first;
        }
        const int s = loads2 % L::kSlots2, n = loads2 / L::kSlots2;
        if (n > 0 && !c.wait(L::kEmpty2 + s, n - 1, 112)) return false;
        const uint32_t to = c.base + L::kOffC + static_cast<uint32_t>(s) * L::kC, full = c.bar(L::kFull2 + s);
        const int col = t2.j * a.bn + half * static_cast<int>(c.rank);
        mbar_arrive_expect_tx(full, c_bytes);
        tma_load_2d_pair(to, &maps.codes, mapa_shared(full, c.rank), col, at2 * 64);
        tma_load_2d_pair(to + L::kCodes, &maps.tiles, mapa_shared(full, c.rank), 0, (col / (4 * kBlock)) * a.chunks + at2 / 2);
        ++loads2;
        if (++at2 == t2.last) at2 = -1, item2 += n_clusters;
        return true;
      };
      bool ok = true;
      for (int i = 0; ok && i < L::kAhead; ++i) ok = next_codes();
#pragma unroll 1
      for (int item = cluster; ok && item < n_items; item += n_clusters) {
        const WgradItem t = wgrad_item(a, item);
        const int col = t.i * 256 + 128 * static_cast<int>(c.rank);
#pragma unroll 1
        for (int st = t.first; st < t.last; ++st) {
          ok = next_codes();
          const int s = loads % L::kSlots, n = loads / L::kSlots;
          ok = ok && loads != most && (n == 0 || c.wait(L::kEmpty + s, n - 1, 111));
          if (!ok) break;
          const uint32_t to = c.base + L::kOffA + static_cast<uint32_t>(s) * L::kA, full = c.lbar(L::kFull + s);
          if (c.leader) mbar_arrive_expect_tx(c.bar(L::kFull + s), 2 * L::kA);
          tma_load_2d_pair(to, &maps.dy, full, 2 * col, st * 64);  // (a map of bytes)
          tma_load_2d_pair(to + 8192, &maps.dy, full, 2 * col + 128, st * 64);
          ++loads;
        }
      }
    }
    __syncwarp();
  } else if (c.warp == L::kMma) {
    if (c.leader) {
      // (64 columns of 64 rows are 8 KB; 8 rows 1 KB)
      const uint64_t ad = sdesc_sw128(c.base + L::kOffA, 8192, 1024), bd = sdesc_sw128(c.base + L::kOffB, 8192, 1024);
      const uint32_t idesc = idesc_wgrad(a.bn);
      bool issued = false, ok = true;
      int load = 0, used = 0;
#pragma unroll 1
      for (int item = cluster; ok && item < n_items; item += n_clusters, ++used) {
        const WgradItem t = wgrad_item(a, item);
        const uint32_t d = c.tmem + 256u * (used & 1);
        if (used >= 2 && !c.wait_all(L::kAccEmpty + (used & 1), (used >> 1) - 1, 113)) break;
#pragma unroll 1
        for (int st = t.first; st < t.last; ++st, ++load) {
          const int s = load % L::kSlots, b = load % L::kSlotsB;
          ok = c.wait_all(L::kFull + s, load / L::kSlots, 114) && c.wait_all(L::kBFull + b, load / L::kSlotsB, 115);
          if (!ok) break;
          issued = true;
          if (elect_one()) {
            tc_fence_after();
            const uint64_t at = ad + static_cast<uint64_t>(s) * (L::kA >> 4), bt = bd + static_cast<uint64_t>(b) * (L::kB >> 4);
#pragma unroll
            for (int q = 0; q < 4; ++q) tc2_mma_ss(d, at + 128 * q, bt + 128 * q, idesc, st > t.first || q > 0 ? 1u : 0u);
            tc2_commit_mc(c.bar(L::kEmpty + s), 3);
            tc2_commit_mc(c.bar(L::kBEmpty + b), 3);
            if (st + 1 == t.last) tc2_commit_mc(c.bar(L::kAccFull + (used & 1)), 3);
          }
          __syncwarp();
        }
      }
      c.finish_mmas(issued);
    }
  } else if (c.warp >= L::kRelay) {
    int total = 0;
    for (int item = cluster; item < n_items; item += n_clusters) {
      const WgradItem t = wgrad_item(a, item);
      total += t.last - t.first;
    }
#pragma unroll 1
    for (int n = c.warp - L::kRelay; n < total; n += 2) {
      const int b = n % L::kSlotsB, k = n / L::kSlotsB;
      if (!c.wait_all(L::kBDone + b, k, 116)) break;
      if (c.leader) {
        if (!c.wait_all(L::kBPeer + b, k, 117) || !__all_sync(0xffffffffu, mbar_try_wait_acquire_cluster(c.bar(L::kBPeer + b), static_cast<uint32_t>(k) & 1u))) break;
        if (c.lane == 0) mbar_arrive(c.bar(L::kBFull + b));
      } else {
        if (c.lane == 0) mbar_arrive_release_cluster(c.lbar(L::kBPeer + b));
      }
      __syncwarp();
    }
  } else if (c.warp >= L::kConvert) {
    // A warp takes four rows at a time, 16 codes a lane (fewer lanes where the tile is narrow).
    const int w = c.warp - L::kConvert, unit = c.lane & 7, sub = c.lane >> 3;
    const bool in = 16 * unit < half;
    int n = 0;
    bool ok = true;
#pragma unroll 1
    for (int item = cluster; ok && item < n_items; item += n_clusters) {
      const WgradItem t = wgrad_item(a, item);
      const int block = (t.j * a.bn + half * static_cast<int>(c.rank)) / kBlock;
#pragma unroll 1
      for (int st = t.first; st < t.last; ++st, ++n) {
        const int s = n % L::kSlots2, b = n % L::kSlotsB;
        ok = c.wait_all(L::kFull2 + s, n / L::kSlots2, 118) && (n < L::kSlotsB || c.wait_all(L::kBEmpty + b, n / L::kSlotsB - 1, 119));
        if (!ok) break;
        const uint8_t* codes = c.ptr + L::kOffC + s * L::kC;
        const uint32_t to = c.base + L::kOffB + static_cast<uint32_t>(b) * L::kB;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const int r = 32 * p + 4 * w + sub;
          const int rt = (st & 1) * 64 + r;  // of the scales' 128 rows
          const uint32_t e = codes[L::kCodes + 16 * (rt & 31) + 4 * (rt >> 5) + (block & 3)];
          // rows past the end hold zeros and anything as scale
          const uint32_t sc = static_cast<int64_t>(st) * 64 + r >= a.rows ? 0u : e == 255u ? 0x7FC0u : e << 7;
          if (in) {
            const uint4 v = *reinterpret_cast<const uint4*>(codes + r * half + 16 * unit);
            const uint2 x0 = codes_to_bf16(v.x, sc * 0x10001u), x1 = codes_to_bf16(v.y, sc * 0x10001u);
            const uint2 x2 = codes_to_bf16(v.z, sc * 0x10001u), x3 = codes_to_bf16(v.w, sc * 0x10001u);
            const uint4 lo = make_uint4(x0.x, x0.y, x1.x, x1.y), hi = make_uint4(x2.x, x2.y, x3.x, x3.y);
            // 64 columns (128 bytes) a row and half of the tile, 16-byte pieces swizzled; the lanes of the
            // second 64 write their odd piece first, so that eight lanes fill all banks
            const uint32_t row = to + (unit >> 2) * 8192u + 128u * r, odd = unit >> 2, piece = 2 * (unit & 3);
            st_shared_v4(row + (((piece + odd) ^ (r & 7)) << 4), odd ? hi : lo);
            st_shared_v4(row + (((piece + 1 - odd) ^ (r & 7)) << 4), odd ? lo : hi);
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (c.lane == 0) {
          mbar_arrive(c.bar(L::kEmpty2 + s));
          mbar_arrive(c.bar(L::kBDone + b));
        }
        __syncwarp();
      }
    }
  } else {
    const int quarter = c.warp;
    int used = 0;
#pragma unroll 1
    for (int item = cluster; item < n_items; item += n_clusters, ++used) {
      const WgradItem t = wgrad_item(a, item);
      const int row = t.i * 256 + 128 * static_cast<int>(c.rank) + 32 * quarter + c.lane, col0 = t.j * a.bn;
      const int cols = row < a.n ? min(a.bn, a.k - col0) : 0;
      const int64_t at = (static_cast<int64_t>(t.part) * a.n + row) * a.k + col0;
      const bool add = a.add != nullptr && a.splits == 1;
      if (!c.wait_all(L::kAccFull + (used & 1), used >> 1, 120)) break;
      tc_fence_after();
      const uint32_t from = c.tmem + 256u * (used & 1) + (static_cast<uint32_t>(quarter) << 21);
#pragma unroll 1
      for (int x = 0; x < a.bn; x += 32) {
        uint32_t r[32];
        tmem_ld32(from + x, r);
        tmem_wait_ld(r);
        if (x + 32 == a.bn) {
          tc_fence_before();
          __syncwarp();
          if (c.lane == 0) mbar_arrive_cluster(c.lbar(L::kAccEmpty + (used & 1)));
        }
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
          if (x + h >= cols) continue;
          if (a.f32) {
            float4* y = reinterpret_cast<float4*>(static_cast<float*>(a.dw) + at + x + h);
            const float4* z = reinterpret_cast<const float4*>(static_cast<const float*>(a.add) + at + x + h);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float4 v = make_float4(__uint_as_float(r[h + 4 * q]), __uint_as_float(r[h + 4 * q + 1]), __uint_as_float(r[h + 4 * q + 2]),
                                     __uint_as_float(r[h + 4 * q + 3]));
              if (add) {
                const float4 o = z[q];
                v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
              }
              y[q] = v;
            }
          } else {
            uint4* y = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.dw) + at + x + h);
            const uint4* z = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.add) + at + x + h);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              Vec8 v;
#pragma unroll
              for (int e = 0; e < 8; ++e) v.v[e] = __uint_as_float(r[h + 8 * q + e]);
              if (add) {
                const Vec8 o = unpack8(z[q]);
#pragma unroll
                for (int e = 0; e < 8; ++e) v.v[e] += o.v[e];
              }
              y[q] = pack8(v);
            }
          }
        }
      }
    }
  }
  c.leave(loads, L::kA, loads2, c_bytes);
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

// d_bias: the sums of dy over the rows.  A cluster of kBiasSplit blocks has 64 columns, eight a thread;
// each block takes every kBiasSplit-th 32 rows, and the first one adds up what the others found, in their order.
constexpr int kBiasSplit = 8;
__global__ void __cluster_dims__(1, kBiasSplit, 1) __launch_bounds__(256) f8_bias_grad_kernel(const uint16_t* dy, int64_t ld, int64_t rows, int n, float* out) {
  __shared__ __align__(16) float part[32][64];
  __shared__ __align__(16) float all[kBiasSplit][64];
  cluster_sync();  // (the others' shared memory is there)
  grid_dependency_wait();
  grid_launch_dependents();
  const int lane = threadIdx.x & 7, sub = threadIdx.x >> 3;
  const int col = blockIdx.x * 64 + 8 * lane, rank = static_cast<int>(cluster_ctarank());
  Vec8 v = fill8(0.f);
  if (col < n) {
#pragma unroll 4
    for (int64_t r = 32 * rank + sub; r < rows; r += 32 * kBiasSplit) {
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
  if (rank == 0 && threadIdx.x < 64 && blockIdx.x * 64 + threadIdx.x < n) {
    float s = 0.f;
    for (int i = 0; i < kBiasSplit; ++i) s += all[i][threadIdx.x];
    out[blockIdx.x * 64 + threadIdx.x] = s;
  }
}

}  // namespace f8
}  // namespace rc
