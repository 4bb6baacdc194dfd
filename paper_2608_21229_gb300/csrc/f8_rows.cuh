// f8_rows.cuh -- rows and weights into their 8-bit form (f8_common.cuh).
#pragma once
#include "f8_common.cuh"

namespace rc {
namespace f8 {

constexpr int kRowsThreads = 256;

// bf16 rows.  A warp takes four strips of 256 columns at a time: eight columns a lane, a block
// to each half of its lanes.  They are of one row, or (kStrips 1, 2: rows of no more strips) of
// as many rows as it takes.  Bound by memory: four loads a lane are on their way together, and the
// four scales of 512 columns are stored as one word.  20608 rows of 4096: 40.8 us, 6.2 TB/s (5 blocks
// an SM that go on to further rows: 42.4; 32 an SM, of which six run at a time, even out the SMs' speeds).
template <int kStrips>
__global__ void __launch_bounds__(kRowsThreads, 6) f8_quantize_kernel(const uint16_t* x, int64_t ld, const Rows out) {
  grid_dependency_wait();
  grid_launch_dependents();
  constexpr int kTall = 4 / kStrips;  // rows at a time
  const int lane = threadIdx.x & 31, parts = (out.width + 256 * kStrips - 1) / (256 * kStrips);  // 1 for kStrips < 4
  const int64_t first = static_cast<int64_t>(blockIdx.x) * (kRowsThreads / 32) + (threadIdx.x >> 5), step = static_cast<int64_t>(gridDim.x) * (kRowsThreads / 32);
  const int64_t step_rows = step / parts * kTall;
  const int step_parts = static_cast<int>(step % parts);
  int64_t row = first / parts * kTall;
  int part = static_cast<int>(first % parts);
  for (; row < out.rows; row += step_rows, part += step_parts) {
    if (part >= parts) part -= parts, ++row;
    if (row >= out.rows) break;
    const int col0 = part * 256 * kStrips + 8 * lane;
    auto row_of = [&](int q) { return row + q / kStrips; };
    auto col_of = [&](int q) { return col0 + 256 * (q % kStrips); };
    auto in = [&](int q) { return col_of(q) < out.width && (kTall == 1 || row_of(q) < out.rows); };
    uint4 raw[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) raw[q] = in(q) ? ld_stream(x + row_of(q) * ld + col_of(q)) : make_uint4(0, 0, 0, 0);
    uint32_t b[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const Vec8 v = unpack8(raw[q]);
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v.v[j]));
#pragma unroll
      for (int d = 1; d < 16; d *= 2) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
      b[q] = scale_byte(m);
      const float s = to_codes(b[q]);
      if (in(q))
        *reinterpret_cast<uint2*>(out.codes + row_of(q) * out.width + col_of(q)) = make_uint2(
            pack_e4m3x4(v.v[0] * s, v.v[1] * s, v.v[2] * s, v.v[3] * s), pack_e4m3x4(v.v[4] * s, v.v[5] * s, v.v[6] * s, v.v[7] * s));
    }
    // Lane 0 has the first block of each strip, lane 16 the second; lane 0 stores the word (or words) of the
    // first two strips, lane 16 that of the others.
    const uint32_t other = __shfl_xor_sync(0xffffffffu, lane < 16 ? b[2] | b[3] << 16 : b[0] | b[1] << 16, 16);
    const uint32_t word = lane < 16 ? b[0] | b[1] << 16 | other << 8 : other | b[2] << 8 | b[3] << 24;
    if ((lane & 15) == 0) {
      const int half = lane >> 4;
      auto put = [&](int64_t r, int group, uint32_t w) {
        if (4 * group >= out.pitch || r >= out.rows) return;
        *reinterpret_cast<uint32_t*>(out.scales + r * out.pitch + 4 * group) = w;
        *reinterpret_cast<uint32_t*>(tile_byte(out, r, 4 * group)) = w;
      };
      if (kStrips == 4) {
        put(row, 2 * part + half, word);
      } else if (kStrips == 2) {
        put(row + half, 0, word);
      } else {
        put(row + 2 * half, 0, word & 0xFFFFu);
        put(row + 2 * half + 1, 0, word >> 16);
      }
    }
  }
}

// A weight [n, k] and its transposed codes: a block of 256 threads takes 128 x 128.
// Warp w holds rows 16 w .. 16 w + 15, four columns a lane, so that a thread has 16
// bytes of four rows of the transposed tile, which go through shared memory into
// whole lines.  Bound by memory, each byte once: fp32 [16384, 4096]: 66 us, 6.1 TB/s; bf16, with half the
// bytes in flight, 65 us, 4.15 TB/s (0.61 of measured).
template <bool kF32>
__global__ void __launch_bounds__(256) f8_quantize_weight_kernel(const void* w, const Rows out, const Rows out_t) {
  __shared__ uint32_t part[8];
  __shared__ __align__(16) uint8_t tile[128 * 128];
  grid_dependency_wait();
  grid_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int r0 = blockIdx.y * 128, c0 = blockIdx.x * 128, n = static_cast<int>(out.rows), k = out.width;
  const int col = c0 + 4 * lane;
  float4 v[16];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int row = r0 + 16 * warp + i;
    v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row < n && col < k) {
      const int64_t at = static_cast<int64_t>(row) * k + col;
      if (kF32) {
        v[i] = __ldcs(reinterpret_cast<const float4*>(static_cast<const float*>(w) + at));
      } else {
        const uint2 t = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(w) + at));
        v[i] = make_float4(__uint_as_float(t.x << 16), __uint_as_float(t.x & 0xFFFF0000u), __uint_as_float(t.y << 16),
                           __uint_as_float(t.y & 0xFFFF0000u));
      }
    }
    m = max(m, max(max(abs_bits(v[i].x), abs_bits(v[i].y)), max(abs_bits(v[i].z), abs_bits(v[i].w))));
  }
  m = __reduce_max_sync(0xffffffffu, m);
  if (lane == 0) part[warp] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, part[i]);
  const uint32_t b = scale_byte(m);
  const float s = to_codes(b);
  uint32_t c[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    c[i] = pack_e4m3x4(v[i].x * s, v[i].y * s, v[i].z * s, v[i].w * s);
    const int row = r0 + 16 * warp + i;
    if (row < n && col < k) *reinterpret_cast<uint32_t*>(out.codes + static_cast<int64_t>(row) * k + col) = c[i];
  }
  if (out_t.codes) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t t[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t lo = __byte_perm(c[4 * q], c[4 * q + 1], (j + 4) << 4 | j), hi = __byte_perm(c[4 * q + 2], c[4 * q + 3], (j + 4) << 4 | j);
        t[q] = __byte_perm(lo, hi, 0x5410);
      }
      // (16-byte pieces of a row in another order for each four rows: no two of a phase share a bank)
      *reinterpret_cast<uint4*>(tile + (4 * lane + j) * 128 + ((warp ^ (lane & 7)) << 4)) = make_uint4(t[0], t[1], t[2], t[3]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * warp + 4 * i + (lane >> 3), ch = lane & 7;  // row of the transposed tile
      const uint4 t = *reinterpret_cast<const uint4*>(tile + r * 128 + ((ch ^ ((r >> 2) & 7)) << 4));
      if (c0 + r < k && r0 + 16 * ch < n) *reinterpret_cast<uint4*>(out_t.codes + static_cast<int64_t>(c0 + r) * n + r0 + 16 * ch) = t;
    }
  }
  if (threadIdx.x == 0) {
    out.scales[static_cast<int64_t>(blockIdx.y) * out.pitch + blockIdx.x] = static_cast<uint8_t>(b);
    if (out_t.codes) out_t.scales[static_cast<int64_t>(blockIdx.x) * out_t.pitch + blockIdx.y] = static_cast<uint8_t>(b);
  }
  if (threadIdx.x < 128) {  // (tiles have room for whole blocks of rows)
    *tile_byte(out, static_cast<int64_t>(r0) + threadIdx.x, blockIdx.x) = static_cast<uint8_t>(b);
    if (out_t.codes) *tile_byte(out_t, static_cast<int64_t>(c0) + threadIdx.x, blockIdx.y) = static_cast<uint8_t>(b);
  }
}

}  // namespace f8
}  // namespace rc
