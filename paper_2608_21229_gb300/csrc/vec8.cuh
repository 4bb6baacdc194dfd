// vec8.cuh -- eight consecutive values of a row as one 16-byte access (bf16) or
// two (fp32), in registers as fp32.
#pragma once
#include <cstdint>

#include "ptx.cuh"

namespace rc {

struct Vec8 {
  float v[8];
};

__device__ __forceinline__ Vec8 unpack8(uint4 r) {
  Vec8 o;
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o.v[2 * i] = __uint_as_float(w[i] << 16);
    o.v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
  return o;
}
__device__ __forceinline__ uint4 pack8(const Vec8& a) {
  return make_uint4(pack_bf16x2(a.v[0], a.v[1]), pack_bf16x2(a.v[2], a.v[3]), pack_bf16x2(a.v[4], a.v[5]),
                    pack_bf16x2(a.v[6], a.v[7]));
}
__device__ __forceinline__ Vec8 fill8(float x) {
  Vec8 o;
#pragma unroll
  for (int i = 0; i < 8; ++i) o.v[i] = x;
  return o;
}
// Elements [i, i + 8) of a parameter row held in bf16 or fp32.  Plain loads here and in the
// kernels: one through the read-only path might be moved above the wait for the kernel
// before, which may have written what is read.
__device__ __forceinline__ Vec8 load_param8(const void* p, int64_t i, bool f32) {
  if (f32) {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
    const float4 a = q[0], b = q[1];
    return Vec8{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
  }
  return unpack8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i));
}
// A load of data that is used once.
__device__ __forceinline__ uint4 ld_stream(const void* p) { return __ldcs(static_cast<const uint4*>(p)); }

// The same as four pairs, for the two-lane fp32 operations.
struct Pair8 {
  f32x2 p[4];
};
__device__ __forceinline__ f32x2 splat2(float x) { return make_f32x2(x, x); }
__device__ __forceinline__ Pair8 unpack_pairs(uint4 r) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  Pair8 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o.p[i] = make_f32x2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  return o;
}
__device__ __forceinline__ uint4 pack_pairs(const Pair8& a) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    split_f32x2(a.p[i], lo, hi);
    w[i] = pack_bf16x2(lo, hi);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ Pair8 pairs_of(const Vec8& a) {
  Pair8 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o.p[i] = make_f32x2(a.v[2 * i], a.v[2 * i + 1]);
  return o;
}
__device__ __forceinline__ float sum2(f32x2 a) {
  float lo, hi;
  split_f32x2(a, lo, hi);
  return lo + hi;
}

}  // namespace rc
