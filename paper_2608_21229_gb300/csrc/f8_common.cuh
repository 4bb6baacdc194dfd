// f8_common.cuh -- the 8-bit form of rows and weights (include/refcache.h): E4M3
// codes and, for each block of 128 columns, a power of two 2^(b - 127) kept as the
// byte b.  The smallest power of two s with amax / s <= 448, so that x / s is
// exact and a code's only error is its rounding: at most 2^-4 of the value, or
// 2^-10 s below E4M3's normal range.  A power of two costs no accuracy against a
// scale of amax / 448 (E4M3 is a floating format), lets the tensor core apply it
// (UE8M0, kind::mxf8f6f4) and makes a decoded value exact in bf16.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "ptx.cuh"
#include "vec8.cuh"

namespace rc {
namespace f8 {

constexpr int kBlock = 128;  // columns of a scale

struct Rows {  // refcache_f8_rows_t, or one orientation of a weight
  uint8_t* codes;
  uint8_t* scales;
  uint8_t* tiles;
  int64_t rows;
  int32_t width, pitch;  // bytes between rows of scales
  int32_t chunks;        // of 128 rows
};
// The scales are kept twice, by rows for those who read the values (weight gradients,
// the GELU's gradient, a caller) and in the order that tcgen05.cp takes, 512 bytes
// for 128 rows and 512 columns, which TMA brings in as they are.  Laid out by a warp
// of the product's kernel instead, the words of 512 columns took 3200 cycles, longer than
// their MMAs (2048).  The byte of a row's block in that order:
__device__ __forceinline__ uint8_t* tile_byte(const Rows& r, int64_t row, int block) {
  return r.tiles + (static_cast<int64_t>(block >> 2) * r.chunks + (row >> 7)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}
__device__ __forceinline__ void put_scale(const Rows& r, int64_t row, int block, uint32_t b) {
  r.scales[row * r.pitch + block] = static_cast<uint8_t>(b);
  *tile_byte(r, row, block) = static_cast<uint8_t>(b);
}

// The largest magnitude of a block is found as the largest of the bits without their
// sign: above every finite value's lie infinity's, above these a NaN's.
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
// b of a block.  255 (UE8M0's NaN) where it holds an infinity or a NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  if (amax >= 0x7F800000u) return 255u;
  if (amax == 0) return 127u;
  // amax = 1.m 2^(e - 127), 448 = 1.75 2^8
  const int b = static_cast<int>(amax >> 23) - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return static_cast<uint32_t>(b < 1 ? 1 : b);
}
// 1 / s; NaN for b = 255, which makes every code of the block a NaN.
__device__ __forceinline__ float to_codes(uint32_t b) { return __uint_as_float(b == 255u ? 0x7FFFFFFFu : (254u - b) << 23); }
__device__ __forceinline__ float from_codes(uint32_t b) { return __uint_as_float(b == 255u ? 0x7FFFFFFFu : b << 23); }

// Four codes as floats (exact).
__device__ __forceinline__ float4 unpack_e4m3x4(uint32_t c) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"(static_cast<uint16_t>(c)));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"(static_cast<uint16_t>(c >> 16)));
  const float2 a = __half22float2(*reinterpret_cast<__half2*>(&lo)), b = __half22float2(*reinterpret_cast<__half2*>(&hi));
  return make_float4(a.x, a.y, b.x, b.y);
}

// ---------------------------------------------------------------- GELU
enum Gelu { kErf = 0, kTanh = 1 };
constexpr float kTanhA = 0.7978845608028654f, kTanhB = 0.044715f;  // sqrt(2 / pi)

// With phi the normal distribution function (or its tanh form, 1 / (1 + exp(-2 z)),
// z = sqrt(2 / pi) (u + 0.044715 u^3)): gelu(u) = u phi, and its derivative.  (Both forms
// keep their relative precision far below zero, where 1 + erf and 1 + tanh cancel: a
// block of nothing but such values has a scale of its own.)
template <int kForm>
__device__ __forceinline__ float gelu(float u) {
  if (kForm == kErf) return 0.5f * u * erfcf(u * -0.7071067811865476f);
  const float z2 = u * (2.0f * kTanhA + 2.0f * kTanhA * kTanhB * u * u);
  return __fdividef(u, 1.0f + __expf(-z2));
}
template <int kForm>
__device__ __forceinline__ float gelu_grad(float u) {
  if (kForm == kErf)
    return 0.5f * erfcf(u * -0.7071067811865476f) + u * __expf(-0.5f * u * u) * 0.3989422804014327f;
  const float z2 = u * (2.0f * kTanhA + 2.0f * kTanhA * kTanhB * u * u);
  const float p = __fdividef(1.0f, 1.0f + __expf(-z2));
  return p + u * p * (1.0f - p) * (2.0f * kTanhA + 6.0f * kTanhA * kTanhB * u * u);
}

// ---------------------------------------------------------------- what becomes of a product
enum Epilogue { kStore = 0, kGelu = 2, kGeluGrad = 4 };  // + the form of the GELU

struct Out {
  const void* bias;  // [width] or null
  int32_t bias_f32;
  int32_t width;  // columns
  int64_t rows;
  uint16_t* y;  // bf16, ld elements between rows (may be null for kGeluGrad)
  int64_t ld;
  Rows a;  // kGelu: the activation; kGeluGrad: the gradient (codes may be null)
  Rows u;  // kGelu: its argument (codes may be null); kGeluGrad: read
};

__device__ __forceinline__ float bias_at(const Out& o, int col) {
  return o.bias_f32 ? static_cast<const float*>(o.bias)[col]
                    : __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(o.bias)[col]) << 16);
}

// One row's block of 128 columns held by a warp, four consecutive columns a lane.
__device__ __forceinline__ void quantize_warp(const Rows& r, int64_t row, int col, bool in, float4 v, int lane) {
  uint32_t m = in ? max(max(abs_bits(v.x), abs_bits(v.y)), max(abs_bits(v.z), abs_bits(v.w))) : 0u;
  m = __reduce_max_sync(0xffffffffu, m);
  const uint32_t b = scale_byte(m);
  const float s = to_codes(b);
  if (in) *reinterpret_cast<uint32_t*>(r.codes + row * r.width + col) = pack_e4m3x4(v.x * s, v.y * s, v.z * s, v.w * s);
  if (lane == 0) put_scale(r, row, col / kBlock, b);
}
template <int kEpi>
__device__ __forceinline__ void finish_row(const Out& o, int64_t row, int col0, int lane, float4 v) {
  const int col = col0 + 4 * lane;
  const bool in = col < o.width;  // (widths are multiples of 16)
  if (o.bias && in) v.x += bias_at(o, col), v.y += bias_at(o, col + 1), v.z += bias_at(o, col + 2), v.w += bias_at(o, col + 3);
  if (kEpi == kStore) {
    if (in) *reinterpret_cast<uint2*>(o.y + row * o.ld + col) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    return;
  }
  if ((kEpi & ~1) == kGelu) {
    if (o.u.codes) quantize_warp(o.u, row, col, in, v, lane);
    v = make_float4(gelu<kEpi & 1>(v.x), gelu<kEpi & 1>(v.y), gelu<kEpi & 1>(v.z), gelu<kEpi & 1>(v.w));
    quantize_warp(o.a, row, col, in, v, lane);
    return;
  }
  if (in) {
    const float4 u = unpack_e4m3x4(*reinterpret_cast<const uint32_t*>(o.u.codes + row * o.u.width + col));
    const float s = from_codes(o.u.scales[row * o.u.pitch + col / kBlock]);
    v.x *= gelu_grad<kEpi & 1>(u.x * s), v.y *= gelu_grad<kEpi & 1>(u.y * s);
    v.z *= gelu_grad<kEpi & 1>(u.z * s), v.w *= gelu_grad<kEpi & 1>(u.w * s);
    if (o.y) *reinterpret_cast<uint2*>(o.y + row * o.ld + col) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
  }
  if (o.a.codes) quantize_warp(o.a, row, col, in, v, lane);
}

}  // namespace f8
}  // namespace rc
