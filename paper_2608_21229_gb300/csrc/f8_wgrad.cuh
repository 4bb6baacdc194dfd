// f8_wgrad.cuh -- a weight's gradient, dw = add + dy^T x, from bf16 dy [rows, n] and x [rows, k]
// in its 8-bit form: bf16 tcgen05 MMAs over CTA pairs, 256 columns of x times 256 (or 128) of
// dy a tile.
//
// The sum runs over the rows, along which x has a scale each, so the tensor core cannot
// apply them.  A code times its power of two is exact in bf16: eight warps of each CTA turn 64
// rows of codes into bf16 in tensor memory, where the MMAs take x from as their first
// operand, and the product is that of dy and of the values that x stands for.
//
// CTA r of a pair holds columns [128 r, 128 r + 128) of x's tile, one block of scales, and half
// of dy's.  A stage is 64 rows: 16 KB of dy, as it lies (MN-major), 8 KB of codes and their
// 512 bytes of scales, which a warp spreads to one bf16 a row.  ldmatrix on bytes with
// transposition gives a thread four rows of one column, whose eight bytes of bf16 are what
// tcgen05.st.16x256b takes from that thread; 64 rows of 16 columns are one such store.
// (Converted in shared memory instead, the second CTA's half had to be released to the first
// one, which issues the MMAs, at cluster scope: 1320 cycles an arrival, and 1180 a stage;
// arrivals that order tensor memory need no such release.)
//
// Tensor memory: 384 columns of sums and four stages of x.  Lane = column of x, so that each store
// of a lane joins those of its warp in one line of dw.  All tiles end at about the same time, and
// what they write waits for the memory, so a tile's sums must not: tiles take columns
// [0, 256) and [128, 384) in turn, eight warps take the 128 columns that both share into
// registers as soon as a tile ends, and the other 128 while the next tile's MMAs run.  Where the
// tiles are few the rows are split and the parts added by another kernel in a fixed order.
#pragma once
#include "f8_pair.cuh"

namespace rc {
namespace f8 {

struct WgradArgs {
  const void* add;   // [n, k] like dw, or null
  void* dw;          // [n, k]; the parts, fp32, where there are several
  int32_t f32;       // dw (and add) fp32, else bf16
  int32_t n, k, bn;  // bn: columns of dy in a tile, 128 or 256
  int64_t rows;
  int32_t chunks;  // of 128 rows
  int32_t stages;  // of 64 rows
  int32_t splits, per_split;  // parts, and stages of each
  Tiles tiles;                // m: of n; n: of k
  Guard guard;
};
struct WgradMaps {
  CUtensorMap dy, codes, tiles;  // 64 rows x 64 columns (128 bytes); 64 rows x 128 columns; 512 bytes
};

struct WgradSmem {
  static constexpr int kSlots = 8, kSlots2 = 8, kSlotsA = 4;  // dy, codes, converted (in tensor memory)
  static constexpr bool kOwn2 = true;  // codes complete on barriers of the CTA that loads them
  static constexpr uint32_t kB = 16384, kCodes = 8192;
  static constexpr uint32_t kOffB = 0, kOffC = kOffB + kSlots * kB, kOffT = kOffC + kSlots2 * kCodes, kOffS = kOffT + kSlots2 * 512,
                            kBars = kOffS + kSlots2 * 128;
  // kFull2, kEmpty2, kScale (a stage's scales are spread) are of each CTA alone; kAccEmpty: the shared sums, the others by turns
  static constexpr int kFull = 0, kEmpty = kFull + kSlots, kFull2 = kEmpty + kSlots, kScale = kFull2 + kSlots2, kEmpty2 = kScale + kSlots2,
                       kAFull = kEmpty2 + kSlots2, kAEmpty = kAFull + kSlotsA, kAccFull = kAEmpty + kSlotsA, kAccEmpty = kAccFull + 1,
                       kDone = kAccEmpty + 3, kNumBars = kDone + 1;
  static constexpr uint32_t kAux = kBars + 8 * kNumBars, kUsed = kAux + 28, kDynamic = kUsed + 1024;
  // warps 0-7: sums; 8-15: codes into bf16, two groups that take turns
  static constexpr int kConvert = 8, kProducer = 16, kMma = 17, kSpread = 18, kProducer2 = 19, kThreads = 32 * 20;
  static constexpr uint32_t kTmemA = 384;
  static_assert(kDynamic <= kMaxDynamic, "shared-memory layout too large");
  __device__ static constexpr uint32_t arrivals(int i) {
    // kEmpty2: the four warps of a group; kAFull: of each CTA; kAccEmpty: eight of each
    return i >= kEmpty2 && i < kAFull ? 4 : i >= kAFull && i < kAEmpty ? 8 : i >= kAccEmpty && i < kDone ? 16 : 1;
  }
};

// Four codes of four rows as bf16, times the rows' scales.  A code's bits shifted to
// bf16's places are its value times 2^-120, E4M3's subnormals being bf16's.
__device__ __forceinline__ void codes_to_bf16(uint32_t c, uint2 scales, uint32_t* to) {
  auto two = [](uint32_t h, uint32_t s) {  // codes in the upper bytes
    const uint32_t v = ((h >> 4) & 0x07F007F0u) | (h & 0x80008000u), up = 0x7B807B80u;  // 2^120
    __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&v);
    x = __hmul2(__hmul2(x, *reinterpret_cast<const __nv_bfloat162*>(&up)), *reinterpret_cast<const __nv_bfloat162*>(&s));
    return *reinterpret_cast<const uint32_t*>(&x);
  };
  to[0] = two(__byte_perm(c, 0, 0x1404), scales.x);
  to[1] = two(__byte_perm(c, 0, 0x3424), scales.y);
}
// Two 16 x 16 tiles of bytes, transposed: r[0], r[1] are rows 4 (lane % 4) .. + 3 of columns
// lane / 4 and lane / 4 + 8 of the first, r[2], r[3] of the second.  Lane l gives row l % 16 of tile l / 16.
__device__ __forceinline__ void ldmatrix_bytes(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// 16 lanes of 32 columns: of each eight columns, a thread has two of lane (lane / 4) and two of that + 8.
__device__ __forceinline__ void tmem_st_16x256(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), "r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
      "r"(r[14]), "r"(r[15])
      : "memory");
}

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

// One lane's column of x, 64 rows of dw (the first `rows` of them there), each a line's part with the
// other lanes'.  What is added comes first, then the sums, then all is stored.
// (The pointers go from row to row: with the rows' addresses kept for the whole tile the registers spill.)
template <typename T>
__device__ __forceinline__ void next_row(T& p, int64_t stride) {
  p += stride;
  asm volatile("" : "+l"(p));
}
template <typename T>
__device__ __forceinline__ void load_rows(float (&v)[64], const T* from, int64_t stride, int rows) {
#pragma unroll
  for (int e = 0; e < 64; ++e) {
    v[e] = 0.f;
    if (e < rows) v[e] = sizeof(T) == 4 ? __uint_as_float(static_cast<uint32_t>(*from)) : __uint_as_float(static_cast<uint32_t>(*from) << 16);
    next_row(from, stride);
  }
}
template <typename T>
__device__ __forceinline__ void store_rows(const float (&v)[64], T* to, int64_t stride, int rows) {
#pragma unroll
  for (int e = 0; e < 64; ++e) {
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
  const int n_items = a.tiles.m * a.tiles.n * a.splits;
  const uint32_t b_bytes = static_cast<uint32_t>(a.bn) * 64u, c_bytes = L::kCodes + 512u;
  int loads = 0, loads2 = 0;
  if (c.warp < L::kConvert) {
    const int group = c.warp >> 2, quarter = c.warp & 3;
    int used = 0;
    bool ok = true;
#pragma unroll 1
    for (int item = cluster; ok && item < n_items; item += n_clusters, ++used) {
      const WgradItem t = wgrad_item(a, item);
      const int col = t.j * 256 + 128 * static_cast<int>(c.rank) + 32 * quarter + c.lane;
      const bool add = a.add != nullptr && a.splits == 1;
      const int turn = used & 1;
#pragma unroll 1
      for (int i = 0; i < 2; ++i) {
        const int h = turn ? i : 1 - i;  // the half in the shared columns first
        const int row0 = t.i * a.bn + 128 * h + 64 * group, rows = col < a.k && 128 * h < a.bn ? a.n - row0 : 0;
        const int64_t at = (static_cast<int64_t>(t.part) * a.n + row0) * a.k + col;
        float v[64];
        if (!add) {
#pragma unroll
          for (int e = 0; e < 64; ++e) v[e] = 0.f;
        } else if (a.f32) {
          load_rows(v, static_cast<const uint32_t*>(a.add) + at, a.k, rows);
        } else {
          load_rows(v, static_cast<const uint16_t*>(a.add) + at, a.k, rows);
        }
        if (i == 0) ok = c.wait_all(L::kAccFull, used, 120);
        if (!ok) break;
        tc_fence_after();
        const uint32_t from = c.tmem + 128u * (turn + h) + 64u * group + (static_cast<uint32_t>(quarter) << 21);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t r[16];
          tmem_ld16(from + 16 * q, r);
          tmem_wait_ld(r);
#pragma unroll
          for (int e = 0; e < 16; ++e) v[16 * q + e] += __uint_as_float(r[e]);
        }
        tc_fence_before();
        __syncwarp();
        if (c.lane == 0) mbar_arrive_cluster(c.lbar(L::kAccEmpty + (i == 0 ? 0 : 1 + turn)));
        if (a.f32)
          store_rows(v, static_cast<uint32_t*>(a.dw) + at, a.k, rows);
        else
          store_rows(v, static_cast<uint16_t*>(a.dw) + at, a.k, rows);
      }
    }
  } else if (c.warp < L::kProducer) {
    const int group = (c.warp - L::kConvert) >> 2, quarter = c.warp & 3;
    const uint32_t lanes = static_cast<uint32_t>(quarter) << 21;
    int n = 0;
    bool ok = true;
#pragma unroll 1
    for (int item = cluster; ok && item < n_items; item += n_clusters) {
      const WgradItem t = wgrad_item(a, item);
#pragma unroll 1
      for (int st = t.first; st < t.last; ++st, ++n) {
        if ((n & 1) != group) continue;
        const int s = n % L::kSlots2, x = n % L::kSlotsA;
        // (the spread scales are there after the codes)
        ok = c.wait_all(L::kScale + s, n / L::kSlots2, 117) && c.wait_all(L::kFull2 + s, n / L::kSlots2, 118) &&
             (n < L::kSlotsA || c.wait_all(L::kAEmpty + x, n / L::kSlotsA - 1, 119));
        if (!ok) break;
        tc_fence_after();
        const uint32_t codes = c.base + L::kOffC + static_cast<uint32_t>(s) * L::kCodes;
        const uint8_t* scales = c.ptr + L::kOffS + s * 128 + 8 * (c.lane & 3);
        uint2 f[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) f[g] = *reinterpret_cast<const uint2*>(scales + 32 * g);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t out[16];
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const int r = 32 * p + c.lane;  // this lane's row of codes, 128 bytes swizzled
            uint32_t v[4];
            ldmatrix_bytes(codes + 128u * r + (((2u * quarter + h) ^ (r & 7)) << 4), v);
#pragma unroll
            for (int e = 0; e < 4; ++e) codes_to_bf16(v[e], f[2 * p + (e >> 1)], out + 8 * p + 2 * e);
          }
          tmem_st_16x256(c.tmem + L::kTmemA + 32u * x + lanes + (static_cast<uint32_t>(h) << 20), out);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (c.lane == 0) {
          mbar_arrive(c.bar(L::kEmpty2 + s));
          mbar_arrive_cluster(c.lbar(L::kAFull + x));
        }
        __syncwarp();
      }
    }
  } else {
    if (c.warp == L::kProducer) {
      if (c.lane == 0) {
        const int most = loads_before_stop(a.guard.stop, c.rank);
        bool ok = true;
#pragma unroll 1
        for (int item = cluster; ok && item < n_items; item += n_clusters) {
          const WgradItem t = wgrad_item(a, item);
          const int col = t.i * a.bn + a.bn / 2 * static_cast<int>(c.rank);
#pragma unroll 1
          for (int st = t.first; st < t.last; ++st) {
            const int s = loads % L::kSlots, n = loads / L::kSlots;
            ok = loads != most && (n == 0 || c.wait(L::kEmpty + s, n - 1, 111));
            if (!ok) break;
            const uint32_t to = c.base + L::kOffB + static_cast<uint32_t>(s) * L::kB, full = c.lbar(L::kFull + s);
            if (c.leader) mbar_arrive_expect_tx(c.bar(L::kFull + s), 2 * b_bytes);
            tma_load_2d_pair(to, &maps.dy, full, 2 * col, st * 64);  // (a map of bytes)
            if (a.bn > 128) tma_load_2d_pair(to + 8192, &maps.dy, full, 2 * col + 128, st * 64);
            ++loads;
          }
        }
      }
      __syncwarp();
    } else if (c.warp == L::kProducer2) {
      if (c.lane == 0) {
        bool ok = true;
#pragma unroll 1
        for (int item = cluster; ok && item < n_items; item += n_clusters) {
          const WgradItem t = wgrad_item(a, item);
          const int col = t.j * 256 + 128 * static_cast<int>(c.rank), line0 = (col / (4 * kBlock)) * a.chunks;
#pragma unroll 1
          for (int st = t.first; st < t.last; ++st) {
            const int s = loads2 % L::kSlots2, n = loads2 / L::kSlots2;
            ok = n == 0 || c.wait(L::kEmpty2 + s, n - 1, 112);
            if (!ok) break;
            const uint32_t bar = c.bar(L::kFull2 + s), full = mapa_shared(bar, c.rank);
            mbar_arrive_expect_tx(bar, c_bytes);
            tma_load_2d_pair(c.base + L::kOffC + static_cast<uint32_t>(s) * L::kCodes, &maps.codes, full, col, st * 64);
            tma_load_2d_pair(c.base + L::kOffT + static_cast<uint32_t>(s) * 512u, &maps.tiles, full, 0, line0 + st / 2);
            ++loads2;
          }
        }
      }
      __syncwarp();
    } else if (c.warp == L::kMma) {
      if (c.leader) {
        const uint64_t bd = sdesc_sw128(c.base + L::kOffB, 8192, 1024);  // (64 columns of 64 rows are 8 KB; 8 rows 1 KB)
        const uint32_t idesc = idesc_bf16_f32(256, a.bn, true);
        bool issued = false, ok = true;
        int load = 0, used = 0;
#pragma unroll 1
        for (int item = cluster; ok && item < n_items; item += n_clusters, ++used) {
          const WgradItem t = wgrad_item(a, item);
          const uint32_t d = c.tmem + 128u * (used & 1);
#pragma unroll 1
          for (int st = t.first; st < t.last; ++st, ++load) {
            const int s = load % L::kSlots, x = load % L::kSlotsA;
            ok = c.wait_all(L::kFull + s, load / L::kSlots, 114) && c.wait_all(L::kAFull + x, load / L::kSlotsA, 115);
            if (ok && st == t.first)
              ok = (used < 1 || c.wait_all(L::kAccEmpty, used - 1, 113)) && (used < 2 || c.wait_all(L::kAccEmpty + 1 + (used & 1), (used >> 1) - 1, 113));
            if (!ok) break;
            issued = true;
            if (elect_one()) {
              tc_fence_after();
              const uint64_t bt = bd + static_cast<uint64_t>(s) * (L::kB >> 4);
              const uint32_t at = c.tmem + L::kTmemA + 32u * x;
#pragma unroll
              for (int q = 0; q < 4; ++q) tc2_mma_ts(d, at + 8u * q, bt + 128 * q, idesc, st > t.first || q > 0 ? 1u : 0u);
              tc2_commit_mc(c.bar(L::kEmpty + s), 3);
              tc2_commit_mc(c.bar(L::kAEmpty + x), 3);
              if (st + 1 == t.last) tc2_commit_mc(c.bar(L::kAccFull), 3);
            }
            __syncwarp();
          }
        }
        c.finish_mmas(issued);
      }
    } else if (c.warp == L::kSpread) {
      // A stage's scales, one bf16 for each of its 64 rows (two a lane).  Rows past the end hold zeros as codes and
      // anything as scale: theirs is 0.
      int n = 0;
      bool ok = true;
#pragma unroll 1
      for (int item = cluster; ok && item < n_items; item += n_clusters) {
        const WgradItem t = wgrad_item(a, item);
        const int block = t.j * 2 + static_cast<int>(c.rank);
#pragma unroll 1
        for (int st = t.first; st < t.last; ++st, ++n) {
          const int s = n % L::kSlots2;
          ok = c.wait_all(L::kFull2 + s, n / L::kSlots2, 116);
          if (!ok) break;
          const uint8_t* tile = c.ptr + L::kOffT + s * 512;
          uint32_t two = 0;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int r = 2 * c.lane + i, rt = (st & 1) * 64 + r;
            const uint32_t e = tile[16 * (rt & 31) + 4 * (rt >> 5) + (block & 3)];
            const uint32_t v = static_cast<int64_t>(st) * 64 + r >= a.rows ? 0u : e == 255u ? 0x7FC0u : e << 7;
            two |= v << (16 * i);
          }
          *reinterpret_cast<uint32_t*>(c.ptr + L::kOffS + s * 128 + 4 * c.lane) = two;
          __syncwarp();
          if (c.lane == 0) mbar_arrive(c.bar(L::kScale + s));
          __syncwarp();
        }
      }
    }
  }
  c.leave(loads, b_bytes, loads2, c_bytes);
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
