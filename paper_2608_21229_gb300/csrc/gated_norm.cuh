// gated_norm.cuh -- the end of one half of a block and the start of the next:
//
//   h = branch, or norm(branch) * post_weight
//   t = x + gate * h                                  (no branch: t = x)
//   y = norm(t) * weight * (1 + scale) + shift        norm: (t - mean) / deviation, or t / rms
//
// with gate, scale and shift of the row's request, and the gradients of that.
// x_out is t rounded to bf16; y comes from t itself.
//
// Bound by memory: forward reads x and the branch and writes x_out and y,
// backward reads x_out, the branch and two gradients and writes two, each once.
// A row is spread over W warps of its block with at most kNV eight-column
// vectors per lane, so that it stays in registers between its statistics and its
// use.  The variance is merged from the threads' own means and sums of squared
// deviations (Chan, Golub and LeVeque's pairwise formula): one exchange instead
// of one for the mean and one for the deviations, and no cancellation where the
// mean is large.
#pragma once
#include "vec8.cuh"

namespace rc {

constexpr int kNormMaxSegs = 64;     // requests of one launch
constexpr int kNormMaxWidth = 8192;
enum : int32_t { kNormNone = 0, kNormLayer = 1, kNormRms = 2 };

struct NormSegs {
  int32_t cu[kNormMaxSegs + 1];  // first row of each request, in rows of the launch
  int32_t n;
};

struct NormArgs {
  const uint16_t *x, *branch;  // backward: x is the stream after the branch (x_out)
  uint16_t *x_out, *y;
  const uint16_t *dy, *dx_out;
  uint16_t *dx, *d_branch;
  const void *gate, *scale, *shift, *weight, *post_weight;
  int64_t ld_gate, ld_scale, ld_shift;  // elements between requests' rows
  float* part;                          // backward: [slot][3][width]
  int32_t rows, width, norm, post_norm, mod_f32;
  int32_t warps_per_row, rows_per_block;
  float eps;
};

__device__ __forceinline__ int segment_of(const NormSegs& s, int row) {
  int lo = 0, hi = s.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.cu[mid] <= row)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// n values with their mean and the sum of their squared deviations.
struct Moments {
  float n, mean, m2;
  __device__ __forceinline__ void merge(float n2, float mean2, float m22) {
    const float total = n + n2;
    const float f = total > 0.f ? __fdividef(n2, total) : 0.f;
    const float d = mean2 - mean;
    mean = fmaf(d, f, mean);
    m2 += m22 + d * d * (n * f);
    n = total;
  }
};

// Statistics of one row (mean, 1 / deviation) over the row's warps.  `slot`: the
// block's shared memory of this exchange, one entry per warp.
template <int kNV>
__device__ __forceinline__ float2 row_stats(const Vec8 (&t)[kNV], int have, int kind, float eps, int width, float4* slot,
                                            int warps, int first_warp) {
  Moments m{8.f * have, 0.f, 0.f};
  float sum = 0.f;
  if (kind == kNormLayer) {
#pragma unroll
    for (int i = 0; i < kNV; ++i)
      if (i < have) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += t[i].v[e];
      }
    m.mean = have ? sum / m.n : 0.f;
  }
#pragma unroll
  for (int i = 0; i < kNV; ++i)
    if (i < have) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = t[i].v[e] - m.mean;
        m.m2 = fmaf(d, d, m.m2);
      }
    }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float n2 = __shfl_xor_sync(0xffffffffu, m.n, o), mean2 = __shfl_xor_sync(0xffffffffu, m.mean, o),
                m22 = __shfl_xor_sync(0xffffffffu, m.m2, o);
    // both lanes of a pair merge the lower one's values first, so that they get the same bits
    const bool upper = (threadIdx.x & o) != 0;
    Moments lo{upper ? n2 : m.n, upper ? mean2 : m.mean, upper ? m22 : m.m2};
    lo.merge(upper ? m.n : n2, upper ? m.mean : mean2, upper ? m.m2 : m22);
    m = lo;
  }
  if (warps > 1) {
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = make_float4(m.n, m.mean, m.m2, 0.f);
    __syncthreads();
    const float4 f = slot[first_warp];
    m = Moments{f.x, f.y, f.z};
    for (int w = 1; w < warps; ++w) {
      const float4 g = slot[first_warp + w];
      m.merge(g.x, g.y, g.z);
    }
  }
  return make_float2(m.mean, rsqrtf(m.m2 / static_cast<float>(width) + eps));
}

// Sums of two values over the row's warps.
__device__ __forceinline__ float2 row_sum2(float a, float b, float4* slot, int warps, int first_warp) {
  a = warp_sum(a);
  b = warp_sum(b);
  if (warps > 1) {
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = make_float4(a, b, 0.f, 0.f);
    __syncthreads();
    a = b = 0.f;
    for (int w = 0; w < warps; ++w) {
      const float4 g = slot[first_warp + w];
      a += g.x;
      b += g.y;
    }
  }
  return make_float2(a, b);
}

template <int kNV>
__global__ void __launch_bounds__(256) gated_norm_kernel(const __grid_constant__ NormSegs segs, const __grid_constant__ NormArgs a) {
  __shared__ float4 slots[2][8];
  const int warps = a.warps_per_row, warp = threadIdx.x >> 5;
  const int group = warp / warps, first_warp = group * warps;
  const int tid = threadIdx.x - 32 * first_warp;
  const int row = blockIdx.x * a.rows_per_block + group;
  const bool on = row < a.rows;
  const int nvec = a.width / 8, stride = 32 * warps;
  const int have = on && tid < nvec ? min(kNV, (nvec - tid + stride - 1) / stride) : 0;
  const bool f32 = a.mod_f32 != 0;
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  const int seg = on ? segment_of(segs, row) : 0;
  const int64_t base = static_cast<int64_t>(on ? row : 0) * a.width;
  Vec8 t[kNV];
  {
    uint4 xr[kNV], br[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      xr[i] = br[i] = make_uint4(0, 0, 0, 0);
      if (i < have) {
        xr[i] = ld_stream(a.x + base + 8 * (tid + i * stride));
        if (a.branch) br[i] = ld_stream(a.branch + base + 8 * (tid + i * stride));
      }
    }
    if (a.branch) {
      Vec8 h[kNV];
#pragma unroll
      for (int i = 0; i < kNV; ++i) h[i] = unpack8(br[i]);
      if (a.post_norm) {
        const float2 st = row_stats<kNV>(h, have, a.post_norm, a.eps, a.width, slots[0], warps, first_warp);
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
          if (i >= have) continue;
          const Vec8 w = a.post_weight ? load_param8(a.post_weight, 8 * (tid + i * stride), f32) : fill8(1.f);
#pragma unroll
          for (int e = 0; e < 8; ++e) h[i].v[e] = (h[i].v[e] - st.x) * st.y * w.v[e];
        }
      }
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        t[i] = unpack8(xr[i]);
        if (i >= have) continue;
        const int col = 8 * (tid + i * stride);
        const Vec8 g = a.gate ? load_param8(a.gate, seg * a.ld_gate + col, f32) : fill8(1.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[i].v[e] = fmaf(g.v[e], h[i].v[e], t[i].v[e]);
        if (a.x_out) *reinterpret_cast<uint4*>(a.x_out + base + col) = pack8(t[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kNV; ++i) t[i] = unpack8(xr[i]);
    }
  }
  if (!a.y) return;
  const float2 st = a.norm ? row_stats<kNV>(t, have, a.norm, a.eps, a.width, slots[1], warps, first_warp) : make_float2(0.f, 1.f);
#pragma unroll
  for (int i = 0; i < kNV; ++i) {
    if (i >= have) continue;
    const int col = 8 * (tid + i * stride);
    const Vec8 w = a.weight ? load_param8(a.weight, col, f32) : fill8(1.f);
    const Vec8 sc = a.scale ? load_param8(a.scale, seg * a.ld_scale + col, f32) : fill8(0.f);
    const Vec8 sh = a.shift ? load_param8(a.shift, seg * a.ld_shift + col, f32) : fill8(0.f);
    Vec8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y.v[e] = fmaf((t[i].v[e] - st.x) * st.y * w.v[e], 1.f + sc.v[e], sh.v[e]);
    *reinterpret_cast<uint4*>(a.y + base + col) = pack8(y);
  }
}

// Backward of one row, with u = dy (1 + scale) weight:
//   d  = dx_out + norm_backward(u),  norm_backward(u) = (u - [mean(u)] - xhat mean(u xhat)) / deviation
//   dx = d,  dh = gate d,  d_branch = dh, or norm_backward(dh post_weight) of the branch's norm
// and the column sums of a request's rows, of which all gradients of
// parameters are made:  A = sum dy,  B = sum dy xhat,  G = sum d fhat (fhat: the
// branch's normalised value before post_weight, or the branch):
//   d_shift = A, d_scale = weight B, d_gate = post_weight G,
//   d_weight = sum over requests (1 + scale) B,  d_post_weight = sum over requests gate G
//
// A block walks over rows_per_block consecutive rows and keeps the three sums of
// its columns in registers; at a request's end they go to slot block + request
// of `part`, which no other (block, request) has.
template <int kNV, int kThreads>
__global__ void __launch_bounds__(kThreads) gated_norm_backward_kernel(const __grid_constant__ NormSegs segs,
                                                                   const __grid_constant__ NormArgs a) {
  __shared__ float4 slots[4][kThreads / 32];
  const int warps = blockDim.x >> 5, tid = threadIdx.x;
  const int nvec = a.width / 8, stride = blockDim.x;
  const int have = tid < nvec ? min(kNV, (nvec - tid + stride - 1) / stride) : 0;
  const bool f32 = a.mod_f32 != 0;
  const int r0 = blockIdx.x * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  Vec8 sa[kNV], sb[kNV], sg[kNV];
#pragma unroll
  for (int i = 0; i < kNV; ++i) sa[i] = sb[i] = sg[i] = fill8(0.f);
  const float inv_w = 1.f / static_cast<float>(a.width);
  int seg = segment_of(segs, r0);
#pragma unroll 1
  for (int row = r0; row < r1; ++row) {
    while (row >= segs.cu[seg + 1]) ++seg;  // (skips requests without rows)
    const int64_t base = static_cast<int64_t>(row) * a.width;
    Vec8 x[kNV], f[kNV];
    uint4 dyr[kNV], dor[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      const int col = 8 * (tid + i * stride);
      const bool on = i < have;
      const uint4 z = make_uint4(0, 0, 0, 0);
      x[i] = unpack8(on && a.dy ? ld_stream(a.x + base + col) : z);
      f[i] = unpack8(on && a.branch ? ld_stream(a.branch + base + col) : z);
      dyr[i] = on && a.dy ? ld_stream(a.dy + base + col) : z;
      dor[i] = on && a.dx_out ? ld_stream(a.dx_out + base + col) : z;
    }
    float2 fs = make_float2(0.f, 1.f);
    if (a.branch && a.post_norm) fs = row_stats<kNV>(f, have, a.post_norm, a.eps, a.width, slots[0], warps, 0);
    Vec8 d[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) d[i] = unpack8(dor[i]);
    if (a.dy) {
      const float2 st = a.norm ? row_stats<kNV>(x, have, a.norm, a.eps, a.width, slots[1], warps, 0) : make_float2(0.f, 1.f);
      Vec8 u[kNV];
      float su = 0.f, sux = 0.f;
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        u[i] = unpack8(dyr[i]);
        if (i >= have) continue;
        const int col = 8 * (tid + i * stride);
        const Vec8 w = a.weight ? load_param8(a.weight, col, f32) : fill8(1.f);
        const Vec8 sc = a.scale ? load_param8(a.scale, seg * a.ld_scale + col, f32) : fill8(0.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[i].v[e] = (x[i].v[e] - st.x) * st.y;
          sa[i].v[e] += u[i].v[e];
          sb[i].v[e] = fmaf(u[i].v[e], x[i].v[e], sb[i].v[e]);
          u[i].v[e] *= (1.f + sc.v[e]) * w.v[e];
          su += u[i].v[e];
          sux = fmaf(u[i].v[e], x[i].v[e], sux);
        }
      }
      float2 s = make_float2(0.f, 0.f);
      if (a.norm) s = row_sum2(su, sux, slots[2], warps, 0);
      const float mu = a.norm == kNormLayer ? s.x * inv_w : 0.f, mux = s.y * inv_w;
#pragma unroll
      for (int i = 0; i < kNV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[i].v[e] = fmaf(st.y, u[i].v[e] - mu - x[i].v[e] * mux, d[i].v[e]);
    }
    float sd = 0.f, sdf = 0.f;
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      if (i >= have) continue;
      const int col = 8 * (tid + i * stride);
      if (a.dx) *reinterpret_cast<uint4*>(a.dx + base + col) = pack8(d[i]);
      if (!a.branch) continue;
      const Vec8 g = a.gate ? load_param8(a.gate, seg * a.ld_gate + col, f32) : fill8(1.f);
      const Vec8 w = a.post_norm && a.post_weight ? load_param8(a.post_weight, col, f32) : fill8(1.f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[i].v[e] = (f[i].v[e] - fs.x) * fs.y;
        sg[i].v[e] = fmaf(d[i].v[e], f[i].v[e], sg[i].v[e]);
        d[i].v[e] *= g.v[e] * w.v[e];
        sd += d[i].v[e];
        sdf = fmaf(d[i].v[e], f[i].v[e], sdf);
      }
    }
    if (a.branch) {
      float mu = 0.f, muf = 0.f;
      if (a.post_norm) {
        const float2 s = row_sum2(sd, sdf, slots[3], warps, 0);
        mu = a.post_norm == kNormLayer ? s.x * inv_w : 0.f;
        muf = s.y * inv_w;
      }
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        if (i >= have) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) d[i].v[e] = fs.y * (d[i].v[e] - mu - f[i].v[e] * muf);
        if (a.d_branch) *reinterpret_cast<uint4*>(a.d_branch + base + 8 * (tid + i * stride)) = pack8(d[i]);
      }
    }
    if (row + 1 == r1 || row + 1 == segs.cu[seg + 1]) {
      float* p = a.part + static_cast<int64_t>(blockIdx.x + seg) * 3 * a.width;
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        if (i >= have) continue;
        const int col = 8 * (tid + i * stride);
        auto put = [&](int k, Vec8& s) {
          float4* q = reinterpret_cast<float4*>(p + static_cast<int64_t>(k) * a.width + col);
          q[0] = make_float4(s.v[0], s.v[1], s.v[2], s.v[3]);
          q[1] = make_float4(s.v[4], s.v[5], s.v[6], s.v[7]);
          s = fill8(0.f);
        };
        put(0, sa[i]);
        put(1, sb[i]);
        put(2, sg[i]);
      }
    }
    __syncthreads();  // the exchange's shared memory is free for the next row
  }
}

struct NormSumArgs {
  const float* part;
  float *d_gate, *d_scale, *d_shift, *d_weight, *d_post_weight;  // [requests, width] and [width], each may be null
  const void *gate, *scale, *weight, *post_weight;
  int64_t ld_gate, ld_scale;
  int32_t width, rows_per_block, mod_f32;
  int32_t add;  // the weights' gradients are added to what an earlier launch left
};

__device__ __forceinline__ float load_param(const void* p, int64_t i, bool f32) {
  return f32 ? static_cast<const float*>(p)[i] : __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(p)[i]) << 16);
}

// The parameters' gradients from the blocks' sums: blockIdx.y = which sum (A, B,
// G); 32 columns by 8 groups that take every eighth slot, joined in a fixed order.
__global__ void __launch_bounds__(256) norm_param_grad_kernel(const __grid_constant__ NormSegs segs, const __grid_constant__ NormSumArgs a) {
  __shared__ float sums[8][33];
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  const int lane = threadIdx.x & 31, g = threadIdx.x >> 5, k = blockIdx.y, col = blockIdx.x * 32 + lane;
  const bool on = col < a.width;
  const bool f32 = a.mod_f32 != 0;
  float total = 0.f;
  for (int s = 0; s < segs.n; ++s) {
    float sum = 0.f;
    if (on && segs.cu[s + 1] > segs.cu[s]) {
      const int b0 = segs.cu[s] / a.rows_per_block, b1 = (segs.cu[s + 1] - 1) / a.rows_per_block;
      const float* p = a.part + (static_cast<int64_t>(s) * 3 + k) * a.width + col;
#pragma unroll 4
      for (int b = b0 + g; b <= b1; b += 8) sum += p[static_cast<int64_t>(b) * 3 * a.width];
    }
    sums[g][lane] = sum;
    __syncthreads();
    if (g == 0 && on) {
      for (int i = 1; i < 8; ++i) sum += sums[i][lane];
      const int64_t at = static_cast<int64_t>(s) * a.width + col;
      if (k == 0) {
        if (a.d_shift) a.d_shift[at] = sum;
      } else if (k == 1) {
        if (a.d_scale) a.d_scale[at] = a.weight ? sum * load_param(a.weight, col, f32) : sum;
        total += (a.scale ? 1.f + load_param(a.scale, s * a.ld_scale + col, f32) : 1.f) * sum;
      } else {
        if (a.d_gate) a.d_gate[at] = a.post_weight ? sum * load_param(a.post_weight, col, f32) : sum;
        total += (a.gate ? load_param(a.gate, s * a.ld_gate + col, f32) : 1.f) * sum;
      }
    }
    __syncthreads();
  }
  float* w = k == 1 ? a.d_weight : k == 2 ? a.d_post_weight : nullptr;
  if (g == 0 && on && w) w[col] = a.add ? w[col] + total : total;
}

}  // namespace rc
