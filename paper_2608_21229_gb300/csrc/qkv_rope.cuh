// qkv_rope.cuh -- from a projection's rows to the attention's q, k and v: per
// head RMS norm of query and key, rotary positions with several axes, rows moved
// to where the packed tensors (or the cache's slots) keep them; and its gradient.
//
//   n = x / sqrt(mean(x^2) + eps) * w          (w absent: n = x)
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t)   for each pair of n, with
//   t = position[axis of the pair] * frequency of the pair
// Gradient, with g the output's gradient turned back by -t and u = g w:
//   dx = r u - x r^3 mean(x u),   r = 1 / sqrt(mean(x^2) + eps);   dw = sum over rows and heads of g x r
//
// The angle is taken in turns: frequency / 2 pi is held as a sum of two fp32
// numbers and the product's whole turns are removed before it is rounded, so
// that the angle is as exact at position 10^6 as at 1 (an fp32 product of
// position and frequency is off by 2^-24 of the whole angle).  sincospif then
// needs no range reduction of its own.
//
// All of it is bound by memory: every head row is read once and written once.  Forward,
// 20608 rows of q, k and v of 24 heads of 128: 120.5 us call after call, 6.3 TB/s.
// A row of one head is 16 bytes for each of D / 8 lanes, so that a warp holds
// 32 / (D / 8) heads of one token at a time, the mean takes log2(D / 8)
// shuffles, and the angles of a token (4 or 8 for each lane) are found once for
// all its heads.
#pragma once
#include "vec8.cuh"

namespace rc {

constexpr int kRopeMaxPairs = 64;
constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = kRopeThreads / 32;  // tokens of a block at a time, one per warp

struct RopeTable {
  float turn_hi[kRopeMaxPairs], turn_lo[kRopeMaxPairs];  // frequency / 2 pi
  uint8_t axis[kRopeMaxPairs];
  int32_t num_axes;
};

struct RopeArgs {
  const uint16_t* src[3];  // forward: q, k, v; backward: q, k and (unused) v
  int64_t ld[3];           // elements between their rows
  uint16_t* dst[3];        // forward: q, k, v out; backward: the gradients of q, k, v
  int64_t ld_dst[3];
  const uint16_t* grad[3];  // backward: gradients of the outputs
  const void* weight[2];    // of q and k, null: not normalised
  const int32_t* positions;
  const int32_t* row_map;  // null: row i is row i of the outputs
  float* dw_part;          // backward: [block][2][D] partial sums of the weights' gradients
  int64_t rows, out_rows;
  int32_t num_heads;
  int32_t weight_f32;
  int32_t head_step;  // heads of a warp's slice (grid.y slices)
  float eps;
};

// The table in shared memory: lanes read different entries of it, which a kernel parameter
// gives one after the other.  (Both kernels fill it before they wait for the one before.
// Without it, and with all eight angles of a lane found by the lane itself, 4608 rows of 24
// heads of 128 took 38 us with pairs in halves, now 29.)
struct RopeShared {
  float4 hi[kRopeMaxPairs / 4], lo[kRopeMaxPairs / 4];
  uint32_t axes[kRopeMaxPairs / 4];  // of four pairs, a byte each
  __device__ __forceinline__ void fill(const RopeTable& t) {
    const int i = threadIdx.x;
    if (i < kRopeMaxPairs) {
      reinterpret_cast<float*>(hi)[i] = t.turn_hi[i];
      reinterpret_cast<float*>(lo)[i] = t.turn_lo[i];
      reinterpret_cast<uint8_t*>(axes)[i] = t.axis[i];
    }
    __syncthreads();
  }
};

// cos and sin of this lane's pairs for one token.  kHalves: lane l of a row
// holds elements [8 l, 8 l + 8), which are the first (l < D / 16) or second
// members of pairs (8 l + e) mod D / 2, so two lanes have the same pairs and find four each;
// else pairs 4 l .. 4 l + 3 whole.
template <int D, bool kHalves>
struct Turn {
  static constexpr int kN = kHalves ? 8 : 4;
  float c[kN], s[kN];
  // position: of axis `lane`, in the first lanes
  __device__ __forceinline__ void set(const RopeShared& t, float position, int l) {
    const bool second = kHalves && l >= D / 16;
    const int at = kHalves ? 2 * (l % (D / 16)) + (second ? 1 : 0) : l;
    const float4 h4 = t.hi[at], l4 = t.lo[at];
    const uint32_t axes = t.axes[at];
    const float hi[4] = {h4.x, h4.y, h4.z, h4.w}, lo[4] = {l4.x, l4.y, l4.z, l4.w};
    float c4[4], s4[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = __shfl_sync(0xffffffffu, position, static_cast<int>((axes >> (8 * e)) & 31u));
      const float whole = p * hi[e];
      const float rest = fmaf(p, hi[e], -whole) + p * lo[e];
      sincospif(2.f * ((whole - rintf(whole)) + rest), &s4[e], &c4[e]);
    }
    if constexpr (kHalves) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float co = __shfl_xor_sync(0xffffffffu, c4[e], D / 16), so = __shfl_xor_sync(0xffffffffu, s4[e], D / 16);
        c[e] = second ? co : c4[e], c[4 + e] = second ? c4[e] : co;
        s[e] = second ? so : s4[e], s[4 + e] = second ? s4[e] : so;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = c4[e], s[e] = s4[e];
    }
  }
  // x turned by the angles (back: by their negatives).
  template <bool kBack>
  __device__ __forceinline__ Vec8 apply(const Vec8& x, int l) const {
    Vec8 o;
    if constexpr (kHalves) {
      const float sign = (l < D / 16) != kBack ? -1.f : 1.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = __shfl_xor_sync(0xffffffffu, x.v[e], D / 16);
        o.v[e] = fmaf(x.v[e], c[e], sign * y * s[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float sn = kBack ? -s[e] : s[e];
        o.v[2 * e] = x.v[2 * e] * c[e] - x.v[2 * e + 1] * sn;
        o.v[2 * e + 1] = x.v[2 * e] * sn + x.v[2 * e + 1] * c[e];
      }
    }
    return o;
  }
};

template <int D>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int o = D / 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// Heads in flight for each tensor: four 16-byte loads a lane.  Four blocks an SM: at three (72
// registers) 4608 rows of 24 heads of 128 take 35.5 us, at four 29.2, at five (51 registers)
// 30.3, and 35.6 with pairs in halves.
template <int D, bool kHalves>
__global__ void __launch_bounds__(kRopeThreads, 4) qkv_rope_kernel(const __grid_constant__ RopeTable table,
                                                                const __grid_constant__ RopeArgs a) {
  constexpr int kLanes = D / 8, kPer = 32 / kLanes, kUnroll = 4;
  const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRopeTokens + (threadIdx.x >> 5);
  __shared__ RopeShared shared;
  shared.fill(table);
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  if (row >= a.rows) return;
  const int64_t to = a.row_map ? a.row_map[row] : row;
  if (to < 0 || to >= a.out_rows) return;
  const int h0 = blockIdx.y * a.head_step, h1 = min(a.num_heads, h0 + a.head_step);
  Turn<D, kHalves> turn;
  if (a.src[0] || a.src[1])
    turn.set(shared, lane < table.num_axes ? static_cast<float>(a.positions[row * table.num_axes + lane]) : 0.f, l);
#pragma unroll 1
  for (int t = 0; t < 3; ++t) {
    if (!a.src[t]) continue;
    const uint16_t* src = a.src[t] + row * a.ld[t] + 8 * l;
    uint16_t* dst = a.dst[t] + to * a.ld_dst[t] + 8 * l;
    const void* wp = t < 2 ? a.weight[t] : nullptr;
    const Vec8 w = wp ? load_param8(wp, 8 * l, a.weight_f32 != 0) : fill8(1.f);
#pragma unroll 1
    for (int h = h0; h < h1; h += kUnroll * kPer) {
      uint4 raw[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int hh = h + u * kPer + sub;
        raw[u] = hh < h1 ? ld_stream(src + hh * D) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int hh = h + u * kPer + sub;
        uint4 out = raw[u];
        if (t < 2) {
          Vec8 x = unpack8(raw[u]);
          if (wp) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(x.v[e], x.v[e], ss);
            const float r = rsqrtf(row_sum<D>(ss) * (1.f / D) + a.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) x.v[e] *= r * w.v[e];
          }
          out = pack8(turn.template apply<false>(x, l));
        }
        if (hh < h1) *reinterpret_cast<uint4*>(dst + hh * D) = out;
      }
    }
  }
}

// The gradient: a warp walks over tokens row, row + stride, ... so that the sums
// of dw stay in registers; the block's sum goes to dw_part.  Bound by the latency of its
// loads, two blocks an SM: 4608 rows of 24 heads of 128 take 42 us, 5.4 TB/s, and
// the sums below 4.  (128 registers a thread; at 80, for three blocks an SM, they spill:
// 67 us.  Loads through a ring in shared memory: 45 us.)
template <int D, bool kHalves>
__global__ void __launch_bounds__(kRopeThreads, 2) qkv_rope_backward_kernel(const __grid_constant__ RopeTable table,
                                                                         const __grid_constant__ RopeArgs a) {
  constexpr int kLanes = D / 8, kPer = 32 / kLanes, kUnroll = 4;
  __shared__ float sums[kRopeTokens][D];
  const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes, warp = threadIdx.x >> 5;
  __shared__ RopeShared shared;
  shared.fill(table);
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  const int h0 = blockIdx.y * a.head_step, h1 = min(a.num_heads, h0 + a.head_step);
  Vec8 w[2], dw[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    w[t] = a.weight[t] ? load_param8(a.weight[t], 8 * l, a.weight_f32 != 0) : fill8(1.f);
    dw[t] = fill8(0.f);
  }
#pragma unroll 1
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * kRopeTokens + warp; row < a.rows;
       row += static_cast<int64_t>(gridDim.x) * kRopeTokens) {
    const int64_t to = a.row_map ? a.row_map[row] : row;
    if (to < 0 || to >= a.out_rows) {  // a row that was not kept has no gradient, whatever it holds
#pragma unroll
      for (int t = 0; t < 3; ++t)
        if (a.grad[t])
          for (int h = h0 + sub; h < h1; h += kPer)
            *reinterpret_cast<uint4*>(a.dst[t] + row * a.ld_dst[t] + h * D + 8 * l) = make_uint4(0, 0, 0, 0);
      continue;
    }
    Turn<D, kHalves> turn;
    if (a.grad[0] || a.grad[1])
      turn.set(shared, lane < table.num_axes ? static_cast<float>(a.positions[row * table.num_axes + lane]) : 0.f, l);
#pragma unroll
    for (int t = 0; t < 3; ++t) {
      if (!a.grad[t]) continue;
      const bool normed = t < 2 && a.weight[t];
      const uint16_t* src = normed ? a.src[t] + row * a.ld[t] + 8 * l : nullptr;
      const uint16_t* grad = a.grad[t] + to * a.num_heads * D + 8 * l;
      uint16_t* dst = a.dst[t] + row * a.ld_dst[t] + 8 * l;
#pragma unroll 1
      for (int h = h0; h < h1; h += kUnroll * kPer) {
        uint4 graw[kUnroll], xraw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int hh = h + u * kPer + sub;
          graw[u] = hh < h1 ? ld_stream(grad + hh * D) : make_uint4(0, 0, 0, 0);
          xraw[u] = normed && hh < h1 ? ld_stream(src + hh * D) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int hh = h + u * kPer + sub;
          uint4 out = graw[u];
          if (t < 2) {
            Vec8 g = turn.template apply<true>(unpack8(graw[u]), l);
            if (normed) {
              const Vec8 x = unpack8(xraw[u]);
              float ss = 0.f, xu = 0.f;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                ss = fmaf(x.v[e], x.v[e], ss);
                xu = fmaf(x.v[e], g.v[e] * w[t < 2 ? t : 0].v[e], xu);
              }
              const float r = rsqrtf(row_sum<D>(ss) * (1.f / D) + a.eps);
              const float k = r * r * r * row_sum<D>(xu) * (1.f / D);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float y = x.v[e];
                if (hh < h1) dw[t < 2 ? t : 0].v[e] = fmaf(g.v[e], y * r, dw[t < 2 ? t : 0].v[e]);
                g.v[e] = fmaf(r, g.v[e] * w[t < 2 ? t : 0].v[e], -y * k);
              }
            }
            out = pack8(g);
          }
          if (hh < h1) *reinterpret_cast<uint4*>(dst + hh * D) = out;
        }
      }
    }
  }
  // the block's sums, lanes of one column first, then warps, in a fixed order
  const int64_t block = static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if (!a.weight[t]) continue;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float s = dw[t].v[e];
#pragma unroll
      for (int o = kLanes; o < 32; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (sub == 0) sums[warp][8 * l + e] = s;
    }
    __syncthreads();
    if (threadIdx.x < D) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < kRopeTokens; ++k) s += sums[k][threadIdx.x];
      a.dw_part[(block * 2 + t) * D + threadIdx.x] = s;
    }
    __syncthreads();
  }
}

// dw = the sum of the blocks' parts, kRopeSumCols columns of one weight a block: 1024 /
// kRopeSumCols groups take every n-th part and are joined in a fixed order.
constexpr int kRopeSumCols = 8;
__global__ void __launch_bounds__(1024) rope_weight_grad_kernel(const float* part, int n_parts, int D, float* dwq,
                                                                float* dwk) {
  __shared__ float sums[32][kRopeSumCols];
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  constexpr int kGroups = 1024 / kRopeSumCols;
  const int t = blockIdx.y, c = threadIdx.x % kRopeSumCols, g = threadIdx.x / kRopeSumCols, col = blockIdx.x * kRopeSumCols + c;
  float* dw = t == 0 ? dwq : dwk;
  if (!dw) return;
  float s = 0.f;
#pragma unroll 4
  for (int i = g; i < n_parts; i += kGroups) s += part[(static_cast<int64_t>(i) * 2 + t) * D + col];
#pragma unroll
  for (int o = kRopeSumCols; o < 32; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) < kRopeSumCols) sums[threadIdx.x >> 5][c] = s;
  __syncthreads();
  if (threadIdx.x < kRopeSumCols) {
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) s += sums[k][c];
    dw[col] = s;
  }
}

}  // namespace rc
