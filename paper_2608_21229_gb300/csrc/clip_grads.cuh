// clip_grads.cuh -- the global norm of many gradient tensors, and the tensors
// scaled so that it is at most max_norm:
//
//   norm = sqrt(sum of squares over all tensors),  out = g * min(1, max_norm / (norm + 1e-6)),
//   out = g for an infinite max_norm
//
// Bound by memory: the tensors are read for the norm, read again to be scaled,
// and written.  The second pass takes the pieces in the opposite order, so that
// what the first read last is still in the L2 (129 MB).  906 M bf16 elements in place: 778
// us, 7.0 TB/s of the two reads and the write (836 with as many pieces for every block).
// Sums are fp32 within a thread's piece, fp64 from there on, and in a fixed order: the
// same tensors give the same bits.
#pragma once
#include "vec8.cuh"

namespace rc {

constexpr int kClipMaxTensors = 512;   // of one launch
constexpr int kClipThreads = 256;
constexpr int kClipPiece = 16384;      // elements a block takes at a time

struct ClipTable {
  const void* g[kClipMaxTensors];
  void* out[kClipMaxTensors];
  int64_t count[kClipMaxTensors];
  int32_t piece0[kClipMaxTensors + 1];  // first piece of each tensor
  uint8_t types[kClipMaxTensors];       // bit 0: gradient fp32, bit 1: output fp32
  int32_t n;
};

struct ClipPiece {
  const uint8_t* src;
  uint8_t* dst;
  int n;
  bool src32, dst32;
};

// The tensor of a piece, from that of a block's piece before it (`lo`, no further than a
// few tensors away, whichever way the block goes).
__device__ __forceinline__ int clip_tensor(const ClipTable& t, int piece, int lo) {
  while (t.piece0[lo + 1] <= piece) ++lo;
  while (t.piece0[lo] > piece) --lo;
  return lo;
}
__device__ __forceinline__ ClipPiece clip_piece(const ClipTable& t, int piece, int lo) {
  const int64_t at = static_cast<int64_t>(piece - t.piece0[lo]) * kClipPiece;
  ClipPiece p;
  p.src32 = (t.types[lo] & 1) != 0;
  p.dst32 = (t.types[lo] & 2) != 0;
  p.src = static_cast<const uint8_t*>(t.g[lo]) + at * (p.src32 ? 4 : 2);
  p.dst = static_cast<uint8_t*>(t.out[lo]) + at * (p.dst32 ? 4 : 2);
  p.n = static_cast<int>(min(static_cast<int64_t>(kClipPiece), t.count[lo] - at));
  return p;
}

__device__ __forceinline__ float clip_load(const uint8_t* p, int i, bool f32) {
  return f32 ? reinterpret_cast<const float*>(p)[i]
             : __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(p)[i]) << 16);
}

// Elements before the first 16-byte boundary (at most n).
__device__ __forceinline__ int clip_head(const uint8_t* p, int size, int n) {
  return min(n, static_cast<int>((16u - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / size);
}

__global__ void __launch_bounds__(kClipThreads) clip_norm_kernel(const __grid_constant__ ClipTable t, double* part, int* taken) {
  __shared__ double sums[kClipThreads / 32];
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x == 0) *taken = 0;
  const int pieces = t.piece0[t.n];
  double total = 0.0;
  int tensor = 0;
  for (int q = blockIdx.x; q < pieces; q += gridDim.x) {
    tensor = clip_tensor(t, q, tensor);
    const ClipPiece p = clip_piece(t, q, tensor);
    const int size = p.src32 ? 4 : 2, per = 16 / size, head = clip_head(p.src, size, p.n);
    const int nv = (p.n - head) / per;
    const uint4* v = reinterpret_cast<const uint4*>(p.src + head * size);
    float s = 0.f;
    if (p.src32) {
#pragma unroll 8
      for (int i = threadIdx.x; i < nv; i += kClipThreads) {
        const uint4 r = v[i];
        const float a = __uint_as_float(r.x), b = __uint_as_float(r.y), c = __uint_as_float(r.z), d = __uint_as_float(r.w);
        s = fmaf(a, a, s), s = fmaf(b, b, s), s = fmaf(c, c, s), s = fmaf(d, d, s);
      }
    } else {
#pragma unroll 8
      for (int i = threadIdx.x; i < nv; i += kClipThreads) {
        const Vec8 r = unpack8(v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(r.v[e], r.v[e], s);
      }
    }
    for (int i = threadIdx.x; i < p.n - nv * per; i += kClipThreads) {
      const float x = clip_load(p.src, i < head ? i : i + nv * per, p.src32);
      s = fmaf(x, x, s);
    }
    total += static_cast<double>(s);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kClipThreads / 32; ++i) total += sums[i];
    part[blockIdx.x] = total;
  }
}

// The scaled tensors of one launch; every block adds up all parts by itself.  `taken`
// counts the pieces taken beyond the blocks' first: SMs run at different speeds.  (Many
// rounds of blocks would even that out too, but each adds the parts up again: with nothing
// to scale, 400 M fp32 elements took 260 us instead of 224.)
__global__ void __launch_bounds__(kClipThreads, 4) clip_scale_kernel(const __grid_constant__ ClipTable t, const double* part, int n_parts,
                                                                  int* taken, float max_norm, float* norm, int in_place) {
  __shared__ double sums[kClipThreads / 32];
  __shared__ int next[2];
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  double total = 0.0;
  for (int i = threadIdx.x; i < n_parts; i += kClipThreads) total += part[i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = total;
  __syncthreads();
  total = 0.0;
  for (int i = 0; i < kClipThreads / 32; ++i) total += sums[i];
  const float nrm = static_cast<float>(sqrt(total));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = nrm;
  const float ratio = max_norm / (nrm + 1e-6f);
  // (an infinite bound bounds nothing, whatever the norm)
  const float coef = !isinf(max_norm) && (ratio < 1.f || isnan(ratio)) ? ratio : 1.f;
  if (in_place && coef == 1.f) return;
  const int pieces = t.piece0[t.n];
  int tensor = max(0, t.n - 1);
  int q = pieces - 1 - static_cast<int>(blockIdx.x);
  for (int k = 0; q >= 0; ++k) {
    if (threadIdx.x == 0) next[k & 1] = pieces - 1 - static_cast<int>(gridDim.x) - atomicAdd(taken, 1);
    tensor = clip_tensor(t, q, tensor);
    const ClipPiece p = clip_piece(t, q, tensor);
    const int size = p.src32 ? 4 : 2, per = 16 / size, head = clip_head(p.src, size, p.n);
    const int nv = (p.n - head) / per;
    const uint4* v = reinterpret_cast<const uint4*>(p.src + head * size);
    uint8_t* dst = p.dst + head * (p.dst32 ? 4 : 2);
    const bool aligned = (reinterpret_cast<uintptr_t>(dst) & 15u) == 0;
    auto put = [&](uint8_t* to, int i, float x) {
      if (p.dst32)
        reinterpret_cast<float*>(to)[i] = x;
      else
        reinterpret_cast<__nv_bfloat16*>(to)[i] = __float2bfloat16_rn(x);
    };
    // eight loads ahead of their stores (which the compiler may not move them over)
    constexpr int kDepth = 8;
#pragma unroll 1
    for (int i0 = threadIdx.x; i0 < nv; i0 += kDepth * kClipThreads) {
      uint4 raw[kDepth];
#pragma unroll
      for (int u = 0; u < kDepth; ++u) {
        const int i = i0 + u * kClipThreads;
        raw[u] = i < nv ? __ldcs(v + i) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < kDepth; ++u) {
        const int i = i0 + u * kClipThreads;
        if (i >= nv) break;
        const uint4 r = raw[u];
        if (p.src32) {
          const float x[4] = {__uint_as_float(r.x) * coef, __uint_as_float(r.y) * coef, __uint_as_float(r.z) * coef,
                              __uint_as_float(r.w) * coef};
          if (p.dst32 && aligned) {
            __stcs(reinterpret_cast<float4*>(dst) + i, make_float4(x[0], x[1], x[2], x[3]));
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) put(dst, 4 * i + e, x[e]);
          }
        } else {
          Vec8 x = unpack8(r);
#pragma unroll
          for (int e = 0; e < 8; ++e) x.v[e] *= coef;
          if (!aligned) {
#pragma unroll
            for (int e = 0; e < 8; ++e) put(dst, 8 * i + e, x.v[e]);
          } else if (p.dst32) {
            __stcs(reinterpret_cast<float4*>(dst) + 2 * i, make_float4(x.v[0], x.v[1], x.v[2], x.v[3]));
            __stcs(reinterpret_cast<float4*>(dst) + 2 * i + 1, make_float4(x.v[4], x.v[5], x.v[6], x.v[7]));
          } else {
            __stcs(reinterpret_cast<uint4*>(dst) + i, pack8(x));
          }
        }
      }
    }
    for (int i = threadIdx.x; i < p.n - nv * per; i += kClipThreads) {
      const int at = i < head ? i : i + nv * per;
      put(p.dst, at, clip_load(p.src, at, p.src32) * coef);
    }
    __syncthreads();
    q = next[k & 1];
  }
}

}  // namespace rc
