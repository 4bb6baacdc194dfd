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
//
// A block walks over a run of consecutive rows, a row spread over all its threads, at
// most kNV eight-column vectors each, which stay in registers between the row's
// statistics and their use.  What the rows of a request share (gate, scale, shift,
// weights) is made into two or three vectors at the request's first row.  The rows
// ahead are on their way into shared memory meanwhile (cp.async; every thread copies
// and reads its own columns, so that no barrier is needed for them): loaded a row at a
// time into registers, a row of 4096 columns took 5 us from its loads to its last
// store, five times its share of the memory's bandwidth.
//
// The mean is found before the squares, from values in registers: two exchanges of the
// block's warps for a layer norm, and no cancellation where the mean is large.
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
  int32_t rows_per_block;
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

// Sums of up to four values over the block's threads; every thread gets them.  Slots
// alternate: two exchanges apart they are free again.
struct BlockSum {
  float4* slots;  // [2][warps]
  int warps, turn = 0;
  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N]) {
    static_assert(N <= 4, "one float4 per warp");
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (warps == 1) return;
    float4* s = slots + turn * warps;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = make_float4(v[0], N > 1 ? v[N > 1 ? 1 : 0] : 0.f, N > 2 ? v[N > 2 ? 2 : 0] : 0.f, N > 3 ? v[N > 3 ? 3 : 0] : 0.f);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
    for (int w = 0; w < warps; ++w) {
      const float4 g = s[w];
      v[0] += g.x;
      if (N > 1) v[N > 1 ? 1 : 0] += g.y;
      if (N > 2) v[N > 2 ? 2 : 0] += g.z;
      if (N > 3) v[N > 3 ? 3 : 0] += g.w;
    }
  }
};

// The rows ahead of the one that is worked on, kTensors of each, in shared memory:
// [slot][tensor][vector][thread], 16 bytes each.
template <int kNV, int kTensors, int kSlots>
struct RowsAhead {
  uint8_t* smem;
  const uint16_t* src[kTensors];  // null: zeros
  int64_t width;
  int have, issued = 0;
  __device__ __forceinline__ uint8_t* at(int slot, int tensor, int i) const {
    return smem + ((static_cast<int64_t>(slot * kTensors + tensor) * kNV + i) * blockDim.x + threadIdx.x) * 16;
  }
  __device__ __forceinline__ void load(int row, bool on) {
    const int slot = issued % kSlots;
    if (on) {
#pragma unroll
      for (int t = 0; t < kTensors; ++t)
        if (src[t]) {
#pragma unroll
          for (int i = 0; i < kNV; ++i)
            if (i < have)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(at(slot, t, i))),
                           "l"(src[t] + row * width + 8 * static_cast<int64_t>(threadIdx.x + i * blockDim.x))
                           : "memory");
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    ++issued;
  }
  // the oldest row that is not read yet: `row`-th of the block
  __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kSlots - 2) : "memory"); }
  __device__ __forceinline__ Vec8 get(int n, int tensor, int i) const {
    if (i >= have || !src[tensor]) return fill8(0.f);
    return unpack8(*reinterpret_cast<const uint4*>(at(n % kSlots, tensor, i)));
  }
};

// (mean, 1 / deviation) of a layer norm, (0, 1 / rms) of an RMS norm.
template <int kNV>
__device__ __forceinline__ float centered_squares(const Vec8 (&t)[kNV], int have, float mean) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kNV; ++i)
    if (i < have) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = t[i].v[e] - mean;
        s = fmaf(d, d, s);
      }
    }
  return s;
}
template <int kNV>
__device__ __forceinline__ float sum_of(const Vec8 (&t)[kNV]) {  // (columns past the row are zero)
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kNV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += t[i].v[e];
  return s;
}
template <int kNV>
__device__ __forceinline__ float2 row_stats(const Vec8 (&t)[kNV], int have, int kind, float eps, float inv_w, BlockSum& sum) {
  float mean = 0.f;
  if (kind == kNormLayer) {
    float s[1] = {sum_of<kNV>(t)};
    sum(s);
    mean = s[0] * inv_w;
  }
  float q[1] = {centered_squares<kNV>(t, have, mean)};
  sum(q);
  return make_float2(mean, rsqrtf(q[0] * inv_w + eps));
}

constexpr int kNormFwdSlots = 4;
// rows of the backward pass in shared memory (four tensors: 64 KB a row at the largest width)
__host__ __device__ constexpr int norm_bwd_slots(int threads) { return threads > 256 ? 2 : 3; }

template <int kNV, int kThreads>
__global__ void __launch_bounds__(kThreads, 512 / kThreads) gated_norm_kernel(const __grid_constant__ NormSegs segs,
                                                                             const __grid_constant__ NormArgs a) {
  extern __shared__ __align__(16) uint8_t smem_norm[];
  __shared__ float4 slots[2 * kThreads / 32];
  const int tid = threadIdx.x, nvec = a.width / 8;
  const int have = tid < nvec ? min(kNV, (nvec - tid + static_cast<int>(blockDim.x) - 1) / static_cast<int>(blockDim.x)) : 0;
  const bool f32 = a.mod_f32 != 0;
  const int r0 = blockIdx.x * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  const float inv_w = 1.f / static_cast<float>(a.width);
  BlockSum sum{slots, static_cast<int>(blockDim.x >> 5)};
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  RowsAhead<kNV, 2, kNormFwdSlots> in{smem_norm, {a.x, a.branch}, a.width, have};
#pragma unroll
  for (int i = 0; i < kNormFwdSlots - 1; ++i) in.load(r0 + i, r0 + i < r1);
  Vec8 gate[kNV], scale[kNV], shift[kNV];  // gate (times the branch's weight), weight (1 + scale), shift
  int seg = segment_of(segs, r0) - 1;
#pragma unroll 1
  for (int row = r0; row < r1; ++row) {
    if (row == r0 || row >= segs.cu[seg + 1]) {
      do ++seg;
      while (row >= segs.cu[seg + 1]);  // (skips requests without rows)
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        if (i >= have) continue;
        const int col = 8 * (tid + i * blockDim.x);
        gate[i] = a.gate ? load_param8(a.gate, seg * a.ld_gate + col, f32) : fill8(1.f);
        const Vec8 pw = a.post_weight ? load_param8(a.post_weight, col, f32) : fill8(1.f);
        const Vec8 w = a.weight ? load_param8(a.weight, col, f32) : fill8(1.f);
        scale[i] = a.scale ? load_param8(a.scale, seg * a.ld_scale + col, f32) : fill8(0.f);
        shift[i] = a.shift ? load_param8(a.shift, seg * a.ld_shift + col, f32) : fill8(0.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          gate[i].v[e] *= pw.v[e];
          scale[i].v[e] = fmaf(w.v[e], scale[i].v[e], w.v[e]);
        }
      }
    }
    in.wait();
    const int n = row - r0;
    const int64_t base = static_cast<int64_t>(row) * a.width;
    Vec8 t[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) t[i] = in.get(n, 0, i);
    if (a.branch) {
      Vec8 h[kNV];
#pragma unroll
      for (int i = 0; i < kNV; ++i) h[i] = in.get(n, 1, i);
      const float2 st = a.post_norm ? row_stats<kNV>(h, have, a.post_norm, a.eps, inv_w, sum) : make_float2(0.f, 1.f);
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        if (i >= have) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) t[i].v[e] = fmaf(gate[i].v[e], (h[i].v[e] - st.x) * st.y, t[i].v[e]);
        if (a.x_out) *reinterpret_cast<uint4*>(a.x_out + base + 8 * (tid + i * blockDim.x)) = pack8(t[i]);
      }
    }
    in.load(row + kNormFwdSlots - 1, row + kNormFwdSlots - 1 < r1);
    if (!a.y) continue;
    const float2 st = a.norm ? row_stats<kNV>(t, have, a.norm, a.eps, inv_w, sum) : make_float2(0.f, 1.f);
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      if (i >= have) continue;
      Vec8 y;
#pragma unroll
      for (int e = 0; e < 8; ++e) y.v[e] = fmaf((t[i].v[e] - st.x) * st.y, scale[i].v[e], shift[i].v[e]);
      *reinterpret_cast<uint4*>(a.y + base + 8 * (tid + i * blockDim.x)) = pack8(y);
    }
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
// A block keeps the three sums of its columns in registers over its rows; at a
// request's end they go to slot block + request of `part`, which no other (block,
// request) has.  The request's two vectors lie in shared memory beside the rows ahead,
// for the registers' sake.
template <int kNV, int kThreads>
__global__ void __launch_bounds__(kThreads, 512 / kThreads) gated_norm_backward_kernel(const __grid_constant__ NormSegs segs,
                                                                                      const __grid_constant__ NormArgs a) {
  constexpr int kSlots = norm_bwd_slots(kThreads);
  extern __shared__ __align__(16) uint8_t smem_norm[];
  __shared__ float4 slots[2 * kThreads / 32];
  const int tid = threadIdx.x, nvec = a.width / 8;
  const int have = tid < nvec ? min(kNV, (nvec - tid + static_cast<int>(blockDim.x) - 1) / static_cast<int>(blockDim.x)) : 0;
  const bool f32 = a.mod_f32 != 0;
  const int r0 = blockIdx.x * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  const float inv_w = 1.f / static_cast<float>(a.width);
  BlockSum sum{slots, static_cast<int>(blockDim.x >> 5)};
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  RowsAhead<kNV, 4, kSlots> in{smem_norm, {a.dy ? a.x : nullptr, a.branch, a.dy, a.dx_out}, a.width, have};
#pragma unroll
  for (int i = 0; i < kSlots - 1; ++i) in.load(r0 + i, r0 + i < r1);
  // [scale or gate][vector][half][thread] float4
  float4* vecs = reinterpret_cast<float4*>(smem_norm + static_cast<int64_t>(kSlots) * 4 * kNV * blockDim.x * 16) + tid;
  auto vec = [&](int k, int i, int h) -> float4& { return vecs[((k * kNV + i) * 2 + h) * blockDim.x]; };
  auto get_vec = [&](int k, int i) -> Vec8 {
    const float4 p = vec(k, i, 0), q = vec(k, i, 1);
    return Vec8{{p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w}};
  };
  Vec8 sa[kNV], sb[kNV], sg[kNV];
#pragma unroll
  for (int i = 0; i < kNV; ++i) sa[i] = sb[i] = sg[i] = fill8(0.f);
  int seg = segment_of(segs, r0) - 1;
#pragma unroll 1
  for (int row = r0; row < r1; ++row) {
    if (row == r0 || row >= segs.cu[seg + 1]) {
      do ++seg;
      while (row >= segs.cu[seg + 1]);  // (skips requests without rows)
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        if (i >= have) continue;
        const int col = 8 * (tid + i * blockDim.x);
        const Vec8 w = a.weight ? load_param8(a.weight, col, f32) : fill8(1.f);
        const Vec8 sc = a.scale ? load_param8(a.scale, seg * a.ld_scale + col, f32) : fill8(0.f);
        const Vec8 g = a.gate ? load_param8(a.gate, seg * a.ld_gate + col, f32) : fill8(1.f);
        const Vec8 pw = a.post_weight ? load_param8(a.post_weight, col, f32) : fill8(1.f);
        float p[8], q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = fmaf(w.v[e], sc.v[e], w.v[e]);
          q[e] = g.v[e] * pw.v[e];
        }
        vec(0, i, 0) = make_float4(p[0], p[1], p[2], p[3]);
        vec(0, i, 1) = make_float4(p[4], p[5], p[6], p[7]);
        vec(1, i, 0) = make_float4(q[0], q[1], q[2], q[3]);
        vec(1, i, 1) = make_float4(q[4], q[5], q[6], q[7]);
      }
    }
    in.wait();
    const int n = row - r0;
    const int64_t base = static_cast<int64_t>(row) * a.width;
    Vec8 x[kNV], f[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      x[i] = in.get(n, 0, i);
      f[i] = in.get(n, 1, i);
    }
    // statistics of both norms in the same exchanges
    const int kind = a.dy ? a.norm : kNormNone, post = a.branch ? a.post_norm : kNormNone;
    float2 xs = make_float2(0.f, 1.f), fs = make_float2(0.f, 1.f);
    if (kind == kNormLayer || post == kNormLayer) {
      float m[2] = {sum_of<kNV>(x), sum_of<kNV>(f)};
      sum(m);
      if (kind == kNormLayer) xs.x = m[0] * inv_w;
      if (post == kNormLayer) fs.x = m[1] * inv_w;
    }
    if (kind || post) {
      float q[2] = {centered_squares<kNV>(x, have, xs.x), centered_squares<kNV>(f, have, fs.x)};
      sum(q);
      if (kind) xs.y = rsqrtf(q[0] * inv_w + a.eps);
      if (post) fs.y = rsqrtf(q[1] * inv_w + a.eps);
    }
    float u2[2] = {0.f, 0.f};
    if (a.dy) {
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        if (i >= have) continue;
        const Vec8 dy = in.get(n, 2, i), w = get_vec(0, i);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[i].v[e] = (x[i].v[e] - xs.x) * xs.y;
          sa[i].v[e] += dy.v[e];
          sb[i].v[e] = fmaf(dy.v[e], x[i].v[e], sb[i].v[e]);
          const float u = dy.v[e] * w.v[e];
          u2[0] += u;
          u2[1] = fmaf(u, x[i].v[e], u2[1]);
        }
      }
      if (kind) sum(u2);
    }
    const float mu = kind == kNormLayer ? u2[0] * inv_w : 0.f, mux = kind ? u2[1] * inv_w : 0.f;
    float d2[2] = {0.f, 0.f};
    Vec8 d[kNV];  // dh times post_weight, in the end
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      if (i >= have) continue;
      const int col = 8 * (tid + i * blockDim.x);
      d[i] = in.get(n, 3, i);
      if (a.dy) {
        const Vec8 dy = in.get(n, 2, i), w = get_vec(0, i);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[i].v[e] = fmaf(xs.y, fmaf(dy.v[e], w.v[e], -fmaf(x[i].v[e], mux, mu)), d[i].v[e]);
      }
      if (a.dx) *reinterpret_cast<uint4*>(a.dx + base + col) = pack8(d[i]);
      if (!a.branch) continue;
      const Vec8 g = get_vec(1, i);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[i].v[e] = (f[i].v[e] - fs.x) * fs.y;
        sg[i].v[e] = fmaf(d[i].v[e], f[i].v[e], sg[i].v[e]);
        d[i].v[e] *= g.v[e];
        d2[0] += d[i].v[e];
        d2[1] = fmaf(d[i].v[e], f[i].v[e], d2[1]);
      }
    }
    in.load(row + kSlots - 1, row + kSlots - 1 < r1);
    if (a.branch) {
      if (post) sum(d2);
      const float md = post == kNormLayer ? d2[0] * inv_w : 0.f, mdf = post ? d2[1] * inv_w : 0.f;
      if (a.d_branch) {
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
          if (i >= have) continue;
#pragma unroll
          for (int e = 0; e < 8; ++e) d[i].v[e] = fs.y * (d[i].v[e] - fmaf(f[i].v[e], mdf, md));
          *reinterpret_cast<uint4*>(a.d_branch + base + 8 * (tid + i * blockDim.x)) = pack8(d[i]);
        }
      }
    }
    if (row + 1 == r1 || row + 1 == segs.cu[seg + 1]) {
      float* p = a.part + static_cast<int64_t>(blockIdx.x + seg) * 3 * a.width;
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        if (i >= have) continue;
        const int col = 8 * (tid + i * blockDim.x);
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
