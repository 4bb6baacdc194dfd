// f8_simple.cuh -- the weight gradient on 8-bit rows, in fp32 FMAs: tiles of 32 x
// 128 outputs, one warp to four rows, four columns a lane.
#pragma once
#include "f8_common.cuh"

namespace rc {
namespace f8 {

__device__ __forceinline__ float value_of(const Rows& r, int64_t row, int64_t scale_row, int col) {
  const float4 v = unpack_e4m3x4(r.codes[row * r.width + col]);
  return v.x * from_codes(r.scales[scale_row * r.pitch + col / kBlock]);
}

template <class A, class B, class F>
__device__ __forceinline__ void simple_product(int64_t rows, int cols, int64_t len, const A& a, const B& b, const F& finish) {
  __shared__ float sa[32][33];
  __shared__ __align__(16) float sb[32][132];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t r0 = static_cast<int64_t>(blockIdx.y) * 32;
  const int c0 = blockIdx.x * 128;
  float4 acc[4] = {};
  for (int64_t l0 = 0; l0 < len; l0 += 32) {
    for (int i = threadIdx.x; i < 32 * 32; i += 256) {
      const int64_t r = r0 + (i >> 5), l = l0 + (i & 31);
      sa[i >> 5][i & 31] = r < rows && l < len ? a(r, l) : 0.f;
    }
    for (int i = threadIdx.x; i < 128 * 32; i += 256) {
      const int c = c0 + (i >> 5);
      const int64_t l = l0 + (i & 31);
      sb[i & 31][i >> 5] = c < cols && l < len ? b(c, l) : 0.f;
    }
    __syncthreads();
#pragma unroll 8
    for (int l = 0; l < 32; ++l) {
      const float4 y = *reinterpret_cast<const float4*>(&sb[l][4 * lane]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = sa[4 * warp + i][l];
        acc[i].x += x * y.x, acc[i].y += x * y.y, acc[i].z += x * y.z, acc[i].w += x * y.w;
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (r0 + 4 * warp + i < rows) finish(r0 + 4 * warp + i, c0, lane, acc[i]);
}


struct WgradArgs {
  const uint16_t* dy;  // [rows, n], ld elements between rows
  int64_t ld;
  Rows x;
  int32_t n;
  const void* add;  // [n, width of x] like dw, or null
  void* dw;
  int32_t f32;
  float* d_bias;
};

__global__ void __launch_bounds__(256) f8_wgrad_simple_kernel(const WgradArgs a) {
  grid_dependency_wait();
  grid_launch_dependents();
  auto bf = [](uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); };
  simple_product(
      a.n, a.x.width, a.x.rows, [&](int64_t r, int64_t l) { return bf(a.dy[l * a.ld + r]); },
      [&](int c, int64_t l) { return value_of(a.x, l, l, c); },
      [&](int64_t r, int c0, int lane, float4 v) {
        const float e[4] = {v.x, v.y, v.z, v.w};
        for (int j = 0; j < 4; ++j) {
          const int c = c0 + 4 * lane + j;
          if (c >= a.x.width) continue;
          const int64_t at = r * a.x.width + c;
          if (a.f32)
            static_cast<float*>(a.dw)[at] = e[j] + (a.add ? static_cast<const float*>(a.add)[at] : 0.f);
          else
            static_cast<uint16_t*>(a.dw)[at] =
                static_cast<uint16_t>(pack_bf16x2(e[j] + (a.add ? bf(static_cast<const uint16_t*>(a.add)[at]) : 0.f), 0.f));
        }
      });
  if (a.d_bias && blockIdx.x == 0)
    for (int64_t r = blockIdx.y * 32 + (threadIdx.x >> 5); r < a.n && r < blockIdx.y * 32 + 32; r += 8) {
      float s = 0.f;
      for (int64_t l = threadIdx.x & 31; l < a.x.rows; l += 32) s += bf(a.dy[l * a.ld + r]);
      for (int d = 16; d; d /= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
      if ((threadIdx.x & 31) == 0) a.d_bias[r] = s;
    }
}

}  // namespace f8
}  // namespace rc
