// f8_common.cuh -- the 8-bit form of rows and weights (include/refcache.h): E4M3
// codes and, for each block of 128 columns, a power of two 2^(b - 127) kept as the
// byte b.  The smallest power of two s with amax / s <= 448, so that x / s is
// exact and a code's only error is its rounding: at most 2^-4 of the value, or
// 2^-10 s below E4M3's normal range.  A power of two costs no accuracy against a
// scale of amax / 448 (E4M3 is a floating format), lets the tensor core apply it
// (UE8M0, kind::mxf8f6f4) and makes a decoded value exact in bf16, but for its ends: below 2^-126 bf16
// has fewer bits, and the largest code of a block whose amax is 248 x 2^120 or more is 256, which stands for 2^128.
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

// The same for a GELU's argument.  2^128 would be an infinity; at half its size a block with such values has the
// same derivative, 1, 0 or at zero 1/2: its codes that are not zero are 2^110 or more.
__device__ __forceinline__ float argument_from_codes(uint32_t b) { return from_codes(b == 247u ? 246u : b); }

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

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ f32x2 rcp2(f32x2 x) {
  float a, b;
  split_f32x2(x, a, b);
  return make_f32x2(rcp_approx(a), rcp_approx(b));
}
__device__ __forceinline__ f32x2 exp2_2(f32x2 x) {
  float a, b;
  split_f32x2(x, a, b);
  return make_f32x2(ex2_approx(a), ex2_approx(b));
}
__device__ __forceinline__ f32x2 abs2(f32x2 x) { return f32x2{x.v & 0x7FFFFFFF7FFFFFFFull}; }

// The normal distribution's tail Q(x), x >= 0, from e = exp(-x^2 / 2): e t R(t) with t =
// 1 / (1 + 0.3 x).  R by a weighted least-squares fit of Q(x) exp(x^2 / 2) / t over Chebyshev nodes of t up
// to x = 13.5 (relative error 1.5e-7, 1.8e-7 with 0.3 in fp32; the exponent's rounding adds 2^-23 x^2).  1 - erf and
// 1 - tanh lose their relative precision far below zero, where a block of nothing but such
// values has a scale of its own.
__device__ __forceinline__ f32x2 normal_tail(f32x2 x, f32x2 e) {
  const f32x2 t = rcp2(fma_f32x2(x, splat2(0.3f), splat2(1.0f)));
  f32x2 p = fma_f32x2(splat2(0.03593191131949425f), t, splat2(-0.15827666223049164f));
  p = fma_f32x2(p, t, splat2(0.2082076519727707f));
  p = fma_f32x2(p, t, splat2(-0.05539471283555031f));
  p = fma_f32x2(p, t, splat2(0.1294696182012558f));
  p = fma_f32x2(p, t, splat2(0.09963738173246384f));
  p = fma_f32x2(p, t, splat2(0.12079837173223495f));
  p = fma_f32x2(p, t, splat2(0.11962638795375824f));
  return mul_f32x2(mul_f32x2(t, e), p);
}
__device__ __forceinline__ f32x2 bell(f32x2 uu) { return exp2_2(mul_f32x2(uu, splat2(-0.72134752f))); }  // exp(-u^2 / 2)
// 1 / (1 + exp(-2 z)), z = sqrt(2 / pi) (u + 0.044715 u^3): the same distribution's tanh form.
constexpr float kTanhA = 1.5957691216057308f, kTanhB = kTanhA * 0.044715f, kLog2e = 1.4426950408889634f;
__device__ __forceinline__ f32x2 logistic(f32x2 u, f32x2 uu) {
  const f32x2 z = mul_f32x2(u, fma_f32x2(uu, splat2(-kTanhB * kLog2e), splat2(-kTanhA * kLog2e)));
  return rcp2(add_f32x2(exp2_2(z), splat2(1.0f)));
}
// gelu(u) = u phi(u)
template <int kForm>
__device__ __forceinline__ f32x2 gelu(f32x2 u) {
  if (kForm == kTanh) return mul_f32x2(u, logistic(u, mul_f32x2(u, u)));
  // u phi(u) = max(u, 0) - |u| Q(|u|)
  float a, b;
  split_f32x2(u, a, b);
  const f32x2 x = abs2(u), minus = f32x2{x.v | 0x8000000080000000ull};
  return fma_f32x2(minus, normal_tail(x, bell(mul_f32x2(u, u))), make_f32x2(fmaxf(a, 0.f), fmaxf(b, 0.f)));
}
template <int kForm>
__device__ __forceinline__ f32x2 gelu_grad(f32x2 u) {
  f32x2 uu = mul_f32x2(u, u);
  if (kForm == kTanh) {
    // (bounded: q is zero long before, and zero times infinity would be a NaN)
    float a, b;
    split_f32x2(uu, a, b);
    uu = make_f32x2(fminf(a, 1e4f), fminf(b, 1e4f));
    const f32x2 p = logistic(u, uu), q = fma_f32x2(p, f32x2{p.v ^ 0x8000000080000000ull}, p);  // p (1 - p)
    return fma_f32x2(mul_f32x2(u, q), fma_f32x2(uu, splat2(3.0f * kTanhB), splat2(kTanhA)), p);
  }
  // phi(u) is Q(|u|) where u's sign is set (-0 too), else 1 - Q(|u|); and u times the density
  float a, b;
  split_f32x2(u, a, b);
  const f32x2 e = bell(uu);
  const f32x2 phi = add_f32x2(f32x2{normal_tail(abs2(u), e).v ^ (~u.v & 0x8000000080000000ull)},
                              make_f32x2(__float_as_int(a) < 0 ? 0.f : 1.f, __float_as_int(b) < 0 ? 0.f : 1.f));
  return fma_f32x2(mul_f32x2(u, splat2(0.3989422804f)), e, phi);
}

// ---------------------------------------------------------------- what becomes of a product
enum Epilogue { kStore = 0, kStoreLines = 1, kGelu = 2, kGeluGrad = 4 };  // + the form of the GELU

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
    split_f32x2(gelu<kEpi & 1>(make_f32x2(v.x, v.y)), v.x, v.y);
    split_f32x2(gelu<kEpi & 1>(make_f32x2(v.z, v.w)), v.z, v.w);
    quantize_warp(o.a, row, col, in, v, lane);
    return;
  }
  if (in) {
    const float4 u = unpack_e4m3x4(*reinterpret_cast<const uint32_t*>(o.u.codes + row * o.u.width + col));
    const float s = argument_from_codes(o.u.scales[row * o.u.pitch + col / kBlock]);
    split_f32x2(mul_f32x2(make_f32x2(v.x, v.y), gelu_grad<kEpi & 1>(make_f32x2(u.x * s, u.y * s))), v.x, v.y);
    split_f32x2(mul_f32x2(make_f32x2(v.z, v.w), gelu_grad<kEpi & 1>(make_f32x2(u.z * s, u.w * s))), v.z, v.w);
    if (o.y) *reinterpret_cast<uint2*>(o.y + row * o.ld + col) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
  }
  if (o.a.codes) quantize_warp(o.a, row, col, in, v, lane);
}

}  // namespace f8
}  // namespace rc
