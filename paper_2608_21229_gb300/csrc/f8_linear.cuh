// f8_linear.cuh -- y = x w^T on 8-bit rows and weights (f8_common.cuh): block-scaled
// tcgen05 MMAs over CTA pairs, 256 rows x up to 256 columns a tile.
//
// CTA r of a pair holds rows [128 r, 128 r + 128) of x's tile and half of w's; a
// stage is 128 columns of both (32 KB), four MMAs of K = 32.  The scales are applied
// by the tensor core: those of 512 columns come as a load of their own (a word with
// the bytes of four blocks for each row) and go into tensor memory by tcgen05.cp, issued before the
// first MMA that needs them.  Sums stay in tensor memory from the first column to the last, of 16384 at most (kSumBlocks).
//
// What bounds it: a stage of 128 columns of x and 256 x 256 of y takes 570 to 600 cycles, of which 512 are MMAs; in long
// calls the power cap (1.4 to 1.6 GHz); in short ones the last round of tiles.  Two sides of a stage take about as long.  With half
// of its MMAs left out it still took 584: its loads alone, 32 KB a CTA at 56 bytes a cycle.  With half of its loads 581: the MMAs
// with the scales' copies and their ring (the weight gradient, which has no scales, came to 529).  With half of both 501, so that each
// side has a part that does not shrink with its work.  1280 x 12288 x 4096: 42.9 to 48.3 us on different GPUs, 2.7 to 3.0 PFLOP/s (0.71 to 0.79 of
// twice the measured bf16 rate); 20608 x 4096 x 12288: 638 to 684 us, 3.0 to 3.25 PFLOP/s (0.80 to 0.86); 4608 rows, 4096 -> 16384 with
// the GELU's two forms: 215 us (tanh), 227 (erf).  The GELU (1792 x 8192 x 2048: 30 us) is bound by its sums' warps: 13800
// cycles a tile for two 8-bit forms and the GELU of 256 x 256, where the MMAs of 2048 columns take 9100: two warps a sub-partition, whose
// registers leave the latencies of one pair of columns to few others (pairs two, four or eight at a time, step by step, took as long).
//
// Tensor memory: two halves of 128 columns of sums, then the scales' slots.  A tile wider
// than 128 takes both halves, a narrower one every second; a half is free as soon as its
// four warps have its 128 columns in registers, a row's block of 128 to a thread, which
// then finds the block's scale, the GELU or its gradient without another thread's help
// while the MMAs of the next tile run.
#pragma once
#include "f8_pair.cuh"

namespace rc {
namespace f8 {

struct LinearArgs {
  Out o;
  int32_t x_chunks, w_chunks;  // 128 rows each
  int32_t k;                   // columns of x
  int32_t bn;                  // columns of a tile: 64, 128, 192 or 256
  Tiles tiles;
  int32_t n_whole, tail, n_items;  // tiles taken whole; the others in pieces of 64 or 128 columns, of 256; whole tiles and pieces
  Guard guard;
};

struct LinearMaps {
  CUtensorMap x, w, w_tail;        // 128 rows, half a tile's (a piece's) columns; 128 codes
  CUtensorMap x_tiles, w_tiles;    // 512 bytes
};

struct LinearSmem {
  static constexpr int kSlots = 6, kSlots2 = 4;  // stages, scales
  static constexpr uint32_t kA = 16384, kSlot = 2 * kA, kScaleSlot = 3 * 512;
  static constexpr uint32_t kScales = kSlots * kSlot, kBias = kScales + kSlots2 * kScaleSlot, kBars = kBias + 8 * 512;
  static constexpr int kFull = 0, kEmpty = kFull + kSlots, kFull2 = kEmpty + kSlots, kEmpty2 = kFull2 + kSlots2, kAccFull = kEmpty2 + kSlots2,
                       kAccEmpty = kAccFull + 2, kDone = kAccEmpty + 2, kNumBars = kDone + 1;
  static constexpr uint32_t kAux = kBars + 8 * kNumBars, kUsed = kAux + kAuxBytes, kDynamic = kUsed + 1024;
  static constexpr int kProducer = 8, kMma = 9, kProducer2 = 10, kThreads = 32 * 12;  // warps 0-7: sums; 8: loads of x; 10: of w
  static constexpr int kSumRegs = 208, kOtherRegs = 80;  // of 168 at launch
  static_assert(256 * kSumRegs + 128 * kOtherRegs <= kThreads * 168, "more registers than the block has");
  static constexpr uint32_t kTmemScales = 256;                       // 16 columns a slot: four of x's words, eight of w's
  static_assert(kDynamic <= kMaxDynamic, "shared-memory layout too large");
  __device__ static constexpr uint32_t arrivals(int i) { return i >= kAccEmpty && i < kDone ? 8 : 1; }  // four warps of each CTA
};

// A tile, or a piece of one: where whole tiles fill the pairs some times over and leave a few, these are taken
// in pieces, one for each pair, as its last.  (A piece of 64 columns takes 320 cycles for each 128 columns of x, a
// tile 512: plan_linear.  240 tiles, 1280 x 4096 times 4096 x 12288: 45.8 -> 42.9 us; 184 tiles in pieces of 128, 1800 x 2048
// times 2048 x 5872: 28.4 -> 25.4.)
struct LinearItem {
  int i, col0, bn;
};
__device__ __forceinline__ LinearItem linear_item(const LinearArgs& a, int t) {
  LinearItem r;
  int j;
  if (t < a.n_whole) {
    a.tiles.at(t, &r.i, &j);
    r.col0 = j * a.bn, r.bn = a.bn;
  } else {
    const int pieces = a.bn / a.tail, p = t - a.n_whole;
    a.tiles.at(a.n_whole + p / pieces, &r.i, &j);
    r.col0 = j * a.bn + p % pieces * a.tail, r.bn = a.tail;
  }
  return r;
}

// Blocks of 128 columns of x whose products are added up in tensor memory, where an addition cuts off what does not
// fit: the error grows with the number of columns (of y's norm, where the products' signs vary / are all alike: 2.2e-7 / 1.4e-6 at 4096
// columns, 1.2e-6 / 9.8e-6 at 16384, 7.4e-6 / 6.0e-5 at 65536).  Of wider rows (kLong) the sums so far go into registers and are added up
// there, rounded to nearest, so that it grows no further (65536: 1.2e-6 / 9.8e-6; 4608 x 512 x 65536 takes 123.9 us, 123.1 without; 2 x
// 24576 x 65536, few rows, 266, 256).  Every 4096 columns instead would cost three waits of some 1300 cycles in the 76000 of a tile of 16384.
// An instance of its own: with the loop over sets in all of them the registers spill.
constexpr int kSumBlocks = 128;

// One row's block of 128 columns, in a thread as 64 pairs.  Of a block that the width cuts, the columns
// behind its end (where `cols`, a multiple of 16, are there) are zero, as their weights are.
__device__ __forceinline__ void load_block(uint32_t t, int cols, f32x2 (&v)[64]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (32 * i >= cols) break;
    uint32_t r[32];
    tmem_ld32(t + 32 * i, r);
    tmem_wait_ld(r);
#pragma unroll
    for (int j = 0; j < 16; ++j) v[16 * i + j] = make_f32x2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
  }
}
__device__ __forceinline__ void add_block(uint32_t t, int cols, f32x2 (&v)[64]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (16 * i >= cols) break;
    uint32_t r[16];
    tmem_ld16(t + 16 * i, r);
    tmem_wait_ld(r);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[8 * i + j] = add_f32x2(v[8 * i + j], make_f32x2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])));
  }
}
// The first n of 8 pieces of 16 bytes of a thread's row.  Each lane has a row of its own, and half a sector (32
// bytes) at a time is twice the requests to the L2: so two pieces at a time where they begin on 32 bytes.
__device__ __forceinline__ void store_pieces(void* to, const uint4 (&c)[8], int n) {
  uint4* y = static_cast<uint4*>(to);
  auto two = [&](int i) {
    if (i + 1 < n)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(y + i), "r"(c[i].x), "r"(c[i].y), "r"(c[i].z), "r"(c[i].w),
                   "r"(c[i + 1].x), "r"(c[i + 1].y), "r"(c[i + 1].z), "r"(c[i + 1].w)
                   : "memory");
    else if (i < n)
      y[i] = c[i];
  };
  if ((reinterpret_cast<uintptr_t>(to) & 31u) == 0) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) two(i);
  } else {
    if (n > 0) y[0] = c[0];
#pragma unroll
    for (int i = 1; i < 7; i += 2) two(i);
    if (n >= 8) y[7] = c[7];
  }
}
// The first n of 8 pieces of 16 bytes of each of a warp's rows, a row a lane: four lanes exchange theirs first, so that each
// of them has the same 32 bytes of four rows, and together they store a line of one row at a time.  (Stored from its own lane, 32
// bytes of 32 rows at a time, a tile's 256 columns in bf16 take 5400 cycles, 12 bytes a cycle, which bounds products of
// few columns: kLinesMost.  The 8-bit forms of a GELU, 8 % slower this way, go from their own lanes.)  `at`: the first row's place; `rows` of the 32 are there.
__device__ __forceinline__ void store_lines(uint8_t* at, int64_t pitch, int rows, int n, uint4 (&c)[8]) {
  const int lane = threadIdx.x & 31, q = lane & 3;
#pragma unroll
  for (int d = 1; d < 4; d *= 2) {
    const bool upper = q & d;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i & d) continue;
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // of a unit of 32 bytes
        uint4 &lo = c[2 * i + h], &hi = c[2 * (i | d) + h];
        auto swap = [&](uint32_t& x, uint32_t& y) {
          const uint32_t other = __shfl_xor_sync(0xffffffffu, upper ? x : y, d);
          if (upper) x = other; else y = other;
        };
        swap(lo.x, hi.x), swap(lo.y, hi.y), swap(lo.z, hi.z), swap(lo.w, hi.w);
      }
    }
  }
  uint8_t* to = at + (lane - q) * pitch + 32 * q;
  const int left = rows - (lane - q), there = n - 2 * q;
#pragma unroll
  for (int i = 0; i < 4; ++i, to += pitch) {
    if (i >= left) break;
    const uint4 x = c[2 * i], y = c[2 * i + 1];
    if (there > 1 && (reinterpret_cast<uintptr_t>(to) & 31u) == 0) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w), "r"(y.x), "r"(y.y),
                   "r"(y.z), "r"(y.w)
                   : "memory");
    } else {
      if (there > 0) reinterpret_cast<uint4*>(to)[0] = x;
      if (there > 1) reinterpret_cast<uint4*>(to)[1] = y;
    }
  }
}
__device__ __forceinline__ void quantize_block(const Rows& r, int64_t row, int col0, int cols, const f32x2 (&v)[64]) {
  float m[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 64; ++i) {
    float a, b;
    split_f32x2(v[i], a, b);
    m[i & 1] = fmax3_abs_nan(a, b, m[i & 1]);
  }
  const uint32_t b = scale_byte(abs_bits(fmax3_abs_nan(m[0], m[1], 0.f)));
  const f32x2 s = splat2(to_codes(b));
  auto four = [&](int i) {
    float x, y, z, w;
    split_f32x2(mul_f32x2(v[i], s), x, y);
    split_f32x2(mul_f32x2(v[i + 1], s), z, w);
    return pack_e4m3x4(x, y, z, w);
  };
  uint4 c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = make_uint4(four(8 * i), four(8 * i + 2), four(8 * i + 4), four(8 * i + 6));
  store_pieces(r.codes + row * r.width + col0, c, cols / 16);
  put_scale(r, row, col0 / kBlock, b);
}
__device__ __forceinline__ void pack_block(int h, const f32x2 (&v)[64], uint4 (&c)[8]) {  // columns 64 h .. 64 h + 63 in bf16
  auto two = [&](int i) {
    float a, b;
    split_f32x2(v[i], a, b);
    return pack_bf16x2(a, b);
  };
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = make_uint4(two(32 * h + 4 * i), two(32 * h + 4 * i + 1), two(32 * h + 4 * i + 2), two(32 * h + 4 * i + 3));
}
__device__ __forceinline__ void store_block(uint16_t* y, int cols, const f32x2 (&v)[64]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint4 c[8];
    pack_block(h, v, c);
    store_pieces(y + 64 * h, c, cols / 8 - 8 * h);
  }
}
// The same by a whole warp, in lines (row: this lane's).
__device__ __forceinline__ void store_block_lines(const Out& o, int64_t row, int col0, int cols, const f32x2 (&v)[64]) {
  const int64_t row0 = row - static_cast<int>(threadIdx.x & 31);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint4 c[8];
    pack_block(h, v, c);
    store_lines(reinterpret_cast<uint8_t*>(o.y + row0 * o.ld + col0 + 64 * h), 2 * o.ld, static_cast<int>(min(static_cast<int64_t>(32), o.rows - row0)),
                cols / 8 - 8 * h, c);
  }
}
// bias: shared memory, 128 floats; u: the codes of the GELU's argument.
template <int kEpi>
__device__ __forceinline__ void finish_block(const Out& o, int64_t row, int col0, int cols, f32x2 (&v)[64], uint32_t bias, const uint4 (&u)[8], float u_scale) {
  if (kEpi < kGeluGrad && o.bias) {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float4 b = ld_shared_f4(bias + 16u * i);
      v[2 * i] = add_f32x2(v[2 * i], make_f32x2(b.x, b.y));
      v[2 * i + 1] = add_f32x2(v[2 * i + 1], make_f32x2(b.z, b.w));
    }
  }
  if (kEpi == kStore) store_block(o.y + row * o.ld + col0, cols, v);
  if (kEpi == kStoreLines) store_block_lines(o, row, col0, cols, v);
  if ((kEpi & ~1) == kGelu) {
    if (o.u.codes) quantize_block(o.u, row, col0, cols, v);
#pragma unroll
    for (int i = 0; i < 64; ++i) v[i] = gelu<kEpi & 1>(v[i]);
    quantize_block(o.a, row, col0, cols, v);
  }
  if ((kEpi & ~1) == kGeluGrad) {
    const f32x2 s = splat2(u_scale);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t w[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 x = unpack_e4m3x4(w[j]);
        f32x2* p = v + 8 * i + 2 * j;
        p[0] = mul_f32x2(p[0], gelu_grad<kEpi & 1>(mul_f32x2(make_f32x2(x.x, x.y), s)));
        p[1] = mul_f32x2(p[1], gelu_grad<kEpi & 1>(mul_f32x2(make_f32x2(x.z, x.w), s)));
      }
    }
    if (o.y) store_block(o.y + row * o.ld + col0, cols, v);
    if (o.a.codes) quantize_block(o.a, row, col0, cols, v);
  }
}

// Of x: kStoreLines for products of no more columns (20000 rows and 10000 columns of y, from its own lane / in lines: 144 columns 117 / 89 us,
// 528 162 / 132, 1040 219 / 208; 4000 and 8192: 1024 columns 30.4 / 32.3, 1536 40.4 / 42.4; 1280 and 12288: 4096 columns 42.6 / 43.8).  Not a branch of one
// kernel: the other side then took 1.5 to 3.5 % more.
constexpr int kLinesMost = 640;

template <int kEpi, bool kLong>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LinearSmem::kThreads, 1)
    f8_linear_kernel(const __grid_constant__ LinearMaps maps, const __grid_constant__ LinearArgs a) {
  using L = LinearSmem;
  extern __shared__ uint8_t smem_raw[];
  Cta<L> c;
  if (!c.enter(smem_raw, a.guard)) return;
  const int cluster = static_cast<int>(blockIdx.x >> 1), n_clusters = static_cast<int>(gridDim.x >> 1);
  const int n_items = a.n_items, blocks = (a.k + kBlock - 1) / kBlock, sums = kLong ? (blocks + kSumBlocks - 1) / kSumBlocks : 1;
  const bool wide = a.bn > 128;  // a whole tile takes both halves, and a piece the first
  auto bytes = [](int bn) { return make_uint2(L::kA, static_cast<uint32_t>(bn) * 64u); };  // of one CTA's load: x, w
  auto scale_bytes = [](int bn) { return make_uint2(512u, 512u * ((bn + 127) / 128)); };
  int loads = 0, loads2 = 0;
  if (c.warp < L::kProducer) {
    more_registers<L::kSumRegs>();
    const int half = c.warp >> 2, quarter = c.warp & 3;
    const uint32_t bias = c.base + L::kBias + 512u * c.warp;
    int used = 0;
#pragma unroll 1
    for (int t = cluster; t < n_items; t += n_clusters, ++used) {
      const LinearItem item = linear_item(a, t);
      const int in_tile = min(128, item.bn - (wide ? 128 * half : 0));
      if (wide ? in_tile <= 0 : (used & 1) != half) continue;
      const int64_t row = static_cast<int64_t>(item.i) * 256 + 128 * c.rank + 32 * quarter + c.lane;
      const int col0 = item.col0 + (wide ? 128 * half : 0);
      const int cols = min(in_tile, a.o.width - col0);
      const bool in = row < a.o.rows && cols > 0;
      uint4 u[8] = {};
      float u_scale = 0.f;
      if ((kEpi & ~1) == kGeluGrad && in) {
        const uint8_t* from = a.o.u.codes + row * a.o.u.width + col0;
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (16 * q < cols) u[q] = *reinterpret_cast<const uint4*>(from + 16 * q);
        u_scale = argument_from_codes(a.o.u.scales[row * a.o.u.pitch + col0 / kBlock]);
      }
      if (kEpi < kGeluGrad && a.o.bias) {  // four columns a lane
        float b[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) b[q] = 4 * c.lane + q < cols ? bias_at(a.o, col0 + 4 * c.lane + q) : 0.f;
        __syncwarp();  // (the tile before has read its own)
        st_shared_v4(bias + 16u * c.lane, make_uint4(__float_as_uint(b[0]), __float_as_uint(b[1]), __float_as_uint(b[2]), __float_as_uint(b[3])));
        __syncwarp();
      }
      const int before = (wide ? used : used >> 1) * sums;
      const uint32_t from = c.tmem + 128u * half + (static_cast<uint32_t>(quarter) << 21);
      f32x2 v[64];
      int n = 0;
#pragma unroll 1
      for (; n < sums; ++n) {
        if (!c.wait_all(L::kAccFull + half, before + n, 106)) break;
        tc_fence_after();
        if (n == 0)
          load_block(from, in_tile, v);
        else
          add_block(from, in_tile, v);
        tc_fence_before();
        __syncwarp();
        if (c.lane == 0) mbar_arrive_cluster(c.lbar(L::kAccEmpty + half));
      }
      if (n < sums) break;
      // (all lanes of a warp whose first row is there, where they store together)
      if (kEpi == kStoreLines ? row - c.lane < a.o.rows && cols > 0 : in) finish_block<kEpi>(a.o, row, col0, cols, v, bias, u, u_scale);
    }
  } else {
    fewer_registers<L::kOtherRegs>();
    if (c.warp == L::kProducer || c.warp == L::kProducer2) {
      if (c.lane == 0) {
        const bool of_x = c.warp == L::kProducer, arms = of_x && c.leader;
        const int most = of_x ? loads_before_stop(a.guard.stop, c.rank) : 0x7FFFFFFF;
        const uint32_t to = c.base + (of_x ? 0u : L::kA);
        bool ok = true;
#pragma unroll 1
        for (int t = cluster; ok && t < n_items; t += n_clusters) {
          const LinearItem item = linear_item(a, t);
          const CUtensorMap* map = of_x ? &maps.x : t < a.n_whole ? &maps.w : &maps.w_tail;
          const int y = of_x ? item.i * 256 + 128 * static_cast<int>(c.rank) : item.col0 + item.bn / 2 * static_cast<int>(c.rank);
          const uint2 b = bytes(item.bn), b2 = scale_bytes(item.bn);
#pragma unroll 1
          for (int kb = 0; ok && kb < blocks; ++kb) {
            if ((kb & 3) == 0) {
              const int s = loads2 % L::kSlots2, n = loads2 / L::kSlots2, g = kb >> 2;
              ok = n == 0 || c.wait(L::kEmpty2 + s, n - 1, 102);
              if (!ok) break;
              const uint32_t at = c.base + L::kScales + static_cast<uint32_t>(s) * L::kScaleSlot, full = c.lbar(L::kFull2 + s);
              if (arms) mbar_arrive_expect_tx(c.bar(L::kFull2 + s), 2 * (b2.x + b2.y));
              if (of_x) {
                tma_load_2d_pair(at, &maps.x_tiles, full, 0, g * a.x_chunks + y / 128);
              } else {
                const int line = g * a.w_chunks + item.col0 / kBlock;
                tma_load_2d_pair(at + 512, &maps.w_tiles, full, 0, line);
                if (item.bn > 128) tma_load_2d_pair(at + 1024, &maps.w_tiles, full, 0, line + 1);
              }
              ++loads2;
            }
            const int s = loads % L::kSlots, n = loads / L::kSlots;
            ok = loads != most && (n == 0 || c.wait(L::kEmpty + s, n - 1, 101));
            if (!ok) break;
            if (arms) mbar_arrive_expect_tx(c.bar(L::kFull + s), 2 * (b.x + b.y));
            tma_load_2d_pair(to + static_cast<uint32_t>(s) * L::kSlot, map, c.lbar(L::kFull + s), kb * kBlock, y);
            ++loads;
          }
        }
      }
      __syncwarp();
    } else if (c.warp == L::kMma) {
      if (c.leader) {
        const uint64_t ad = sdesc_sw128(c.base, 16, 1024), bd = sdesc_sw128(c.base + L::kA, 16, 1024);
        const uint64_t sd = scales_desc(c.base + L::kScales);
        bool issued = false, ok = true;
        int load = 0, group = 0, used = 0;
#pragma unroll 1
        for (int t = cluster; ok && t < n_items; t += n_clusters, ++used) {
          const LinearItem item = linear_item(a, t);
          const bool both = item.bn > 128;
          const int first = wide ? 0 : used & 1;  // half
          const uint32_t d = c.tmem + 128u * first, idesc = idesc_mx(256, item.bn);
          const uint32_t shift = static_cast<uint32_t>(item.col0 % kBlock) / 32u;  // it may begin in the middle of a chunk
          // the half's (both halves') earlier sums are in registers
          int before = (wide ? used : used >> 1) * sums;
#pragma unroll 1
          for (int kb = 0; kb < blocks; ++kb, ++load) {
            const int in_sum = kLong ? kb % kSumBlocks : kb;
            if (in_sum == 0) {
              ok = before == 0 || (c.wait_all(L::kAccEmpty + first, before - 1, 103) && (!both || c.wait_all(L::kAccEmpty + 1, before - 1, 103)));
              if (!ok) break;
              ++before;
            }
            const int s = load % L::kSlots, sc = group % L::kSlots2;
            const uint32_t sfa = c.tmem + L::kTmemScales + 16u * sc, sfb = sfa + 4;
            if ((kb & 3) == 0) {
              ok = c.wait_all(L::kFull2 + sc, group / L::kSlots2, 104);
              if (!ok) break;
            }
            ok = c.wait_all(L::kFull + s, load / L::kSlots, 105);
            if (!ok) break;
            issued = true;
            const int steps = min(4, (a.k - kb * kBlock + 31) / 32);
            const bool last = kb + 1 == blocks, out = last || (kLong && in_sum == kSumBlocks - 1);
            if (elect_one()) {
              tc_fence_after();
              if ((kb & 3) == 0) {
                const uint64_t at = sd + static_cast<uint64_t>(sc) * (L::kScaleSlot >> 4);
                copy_scales_pair(sfa, at);
                copy_scales_pair(sfb, at + (512 >> 4));
                if (both) copy_scales_pair(sfb + 4, at + (1024 >> 4));
              }
              const uint64_t off = static_cast<uint64_t>(s) * (L::kSlot >> 4);
              const uint32_t id = idesc_byte(idesc, kb & 3);
#pragma unroll
              for (int q = 0; q < 4; ++q)
                if (q < steps) mx_mma_pair(d, ad + off + 2 * q, bd + off + 2 * q, id, sfa, sfb + shift, in_sum > 0 || q > 0 ? 1u : 0u);
              tc2_commit_mc(c.bar(L::kEmpty + s), 3);
              if ((kb & 3) == 3 || last) tc2_commit_mc(c.bar(L::kEmpty2 + sc), 3);
              if (out) {
                tc2_commit_mc(c.bar(L::kAccFull + first), 3);
                if (both) tc2_commit_mc(c.bar(L::kAccFull + 1), 3);
              }
            }
            __syncwarp();
            if ((kb & 3) == 3 || last) ++group;
          }
        }
        c.finish_mmas(issued);
      }
    }
  }
  const int whole = cluster < a.n_whole ? (a.n_whole - cluster + n_clusters - 1) / n_clusters : 0;  // tiles of this pair
  c.leave(Loads{loads, bytes(a.bn), bytes(a.tail), whole * blocks}, Loads{loads2, scale_bytes(a.bn), scale_bytes(a.tail), whole * ((blocks + 3) / 4)});
}

}  // namespace f8
}  // namespace rc
