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
// weights) is made into a few vectors at the request's first row.  The rows ahead are on
// their way into shared memory meanwhile (cp.async; every thread copies and reads its own
// columns, so that no barrier is needed for them).  8704 rows of 4096 columns, layer norm:
// 49 us call after call, 5.8 TB/s; 67.6 when a row was loaded into registers as its turn
// came, since a block waits for memory once a row then.
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

// Sums of a few values over the block's threads; every thread gets them.  Slots
// alternate: two exchanges apart they are free again.
template <int kWarps>
struct BlockSum {
  float4* slots;  // [2][kWarps]
  int turn = 0;
  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N]) {
    static_assert(N <= 2, "two of a float4's values");
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if constexpr (kWarps > 1) {
      float4* s = slots + turn;
      turn ^= kWarps;
      if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = make_float4(v[0], N > 1 ? v[N - 1] : 0.f, 0.f, 0.f);
      __syncthreads();
      // every warp adds up the warps' sums, a lane each
      const float4 g = s[threadIdx.x & (kWarps - 1)];
      v[0] = g.x;
      if (N > 1) v[N - 1] = g.y;
#pragma unroll
      for (int o = 1; o < kWarps; o <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
  }
};

// The rows ahead of the one that is worked on, kTensors of each, in shared memory:
// [slot][tensor][vector][thread], 16 bytes each.  A tensor that is not there (null) and
// a vector past the row's end read as zeros.  Thread t has vectors t and t + kThreads of
// a row; all tensors share one offset into them.
template <int kNV, int kThreads, int kTensors, int kSlots>
struct RowsAhead {
  static constexpr uint32_t kVec = 16u * kThreads, kTensor = kNV * kVec, kSlot = kTensors * kTensor;
  uint8_t* mine;               // this thread's first 16 bytes
  bool last;                   // the kNV-th vector is inside the row
  uint32_t write = 0, read = 0;  // bytes of the slots
  __device__ __forceinline__ void init(uint8_t* smem, const uint16_t* const (&src)[kTensors], bool last_vector) {
    last = last_vector;
    mine = smem + 16u * threadIdx.x;
#pragma unroll
    for (int t = 0; t < kTensors; ++t)
#pragma unroll
      for (int i = 0; i < kNV; ++i)
        if (!src[t] || (i == kNV - 1 && !last)) {
#pragma unroll
          for (int s = 0; s < kSlots; ++s) *reinterpret_cast<uint4*>(mine + s * kSlot + t * kTensor + i * kVec) = make_uint4(0, 0, 0, 0);
        }
  }
  // `off`: bytes from the tensors' start to this thread's first vector of the row
  __device__ __forceinline__ void load(const uint16_t* const (&src)[kTensors], int64_t off, bool on) {
    if (on) {
#pragma unroll
      for (int t = 0; t < kTensors; ++t)
        if (src[t]) {
          const uint8_t* from = reinterpret_cast<const uint8_t*>(src[t]) + off;
          const uint32_t to = smem_u32(mine + write + t * kTensor);
#pragma unroll
          for (int i = 0; i < kNV; ++i)
            if (i < kNV - 1 || last)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + i * kVec), "l"(from + i * kVec) : "memory");
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    write = write + kSlot == kSlots * kSlot ? 0u : write + kSlot;
  }
  __device__ __forceinline__ Pair8 get(int tensor, int i) const {
    return unpack_pairs(*reinterpret_cast<const uint4*>(mine + read + tensor * kTensor + i * kVec));
  }
  __device__ __forceinline__ void next() { read = read + kSlot == kSlots * kSlot ? 0u : read + kSlot; }
};

// Sums over this thread's columns: of the values, and of the squares of their
// distances from the mean (columns past the row are zero, and left out there).
template <int kNV>
__device__ __forceinline__ float sum_of(const Pair8 (&t)[kNV]) {
  f32x2 s = splat2(0.f);
#pragma unroll
  for (int i = 0; i < kNV; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) s = add_f32x2(s, t[i].p[e]);
  return sum2(s);
}
template <int kNV>
__device__ __forceinline__ float centered_squares(const Pair8 (&t)[kNV], float mean, bool last) {
  const f32x2 m = splat2(-mean);
  float total = 0.f;
#pragma unroll
  for (int i = 0; i < kNV; ++i) {
    f32x2 s = splat2(0.f);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x2 d = add_f32x2(t[i].p[e], m);
      s = fma_f32x2(d, d, s);
    }
    total += i < kNV - 1 || last ? sum2(s) : 0.f;
  }
  return total;
}
// (mean, 1 / deviation) of a layer norm, (0, 1 / rms) of an RMS norm.
template <int kNV, typename Sum>
__device__ __forceinline__ float2 row_stats(const Pair8 (&t)[kNV], bool last, int kind, float eps, float inv_w, Sum& sum) {
  float mean = 0.f;
  if (kind == kNormLayer) {
    float s[1] = {sum_of<kNV>(t)};
    sum(s);
    mean = s[0] * inv_w;
  }
  float q[1] = {centered_squares<kNV>(t, mean, last)};
  sum(q);
  return make_float2(mean, rsqrtf(q[0] * inv_w + eps));
}

constexpr int kNormFwdSlots = 4;
// Rows of the backward pass in shared memory (four tensors: 32 KB a row at a width of 4096).
constexpr int kNormBwdSlots = 2;

template <int kNV, int kThreads>
__global__ void __launch_bounds__(kThreads, 512 / kThreads) gated_norm_kernel(const __grid_constant__ NormSegs segs,
                                                                             const __grid_constant__ NormArgs a) {
  extern __shared__ __align__(16) uint8_t smem_norm[];
  __shared__ float4 slots[2 * kThreads / 32];
  const int tid = threadIdx.x;
  const bool last = (tid + (kNV - 1) * kThreads) * 8 < a.width;
  const bool f32 = a.mod_f32 != 0;
  const int r0 = blockIdx.x * a.rows_per_block, r1 = r0 + min(a.rows - r0, a.rows_per_block);  // (the sum of the two may pass 2^31)
  const float inv_w = 1.f / static_cast<float>(a.width);
  BlockSum<kThreads / 32> sum{slots};
  constexpr uint32_t kVec = 16u * kThreads;  // bytes between a thread's vectors
  const int64_t row_bytes = 2 * static_cast<int64_t>(a.width);
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  const uint16_t* const src[2] = {a.x, a.branch};
  RowsAhead<kNV, kThreads, 2, kNormFwdSlots> in;
  in.init(smem_norm, src, last);
  int64_t off = r0 * row_bytes + 16 * tid;  // of this thread's first vector of the row
#pragma unroll
  for (int i = 0; i < kNormFwdSlots - 1; ++i) in.load(src, off + i * row_bytes, r0 + i < r1);
  Pair8 gate[kNV], scale[kNV], shift[kNV];  // gate (times the branch's weight), weight (1 + scale), shift
  int seg = segment_of(segs, r0) - 1, end = r0;
#pragma unroll 1
  for (int row = r0; row < r1; ++row, off += row_bytes) {
    if (row >= end) {
      do end = segs.cu[++seg + 1];
      while (row >= end);  // (skips requests without rows)
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        gate[i] = scale[i] = shift[i] = pairs_of(fill8(0.f));
        if (i == kNV - 1 && !last) continue;
        const int col = 8 * (tid + i * kThreads);
        Vec8 g = a.gate ? load_param8(a.gate, seg * a.ld_gate + col, f32) : fill8(1.f);
        const Vec8 pw = a.post_weight ? load_param8(a.post_weight, col, f32) : fill8(1.f);
        const Vec8 w = a.weight ? load_param8(a.weight, col, f32) : fill8(1.f);
        Vec8 sc = a.scale ? load_param8(a.scale, seg * a.ld_scale + col, f32) : fill8(0.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          g.v[e] *= pw.v[e];
          sc.v[e] = fmaf(w.v[e], sc.v[e], w.v[e]);
        }
        gate[i] = pairs_of(g);
        scale[i] = pairs_of(sc);
        if (a.shift) shift[i] = pairs_of(load_param8(a.shift, seg * a.ld_shift + col, f32));
      }
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(kNormFwdSlots - 2) : "memory");
    Pair8 t[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) t[i] = in.get(0, i);
    if (a.branch) {
      Pair8 h[kNV];
#pragma unroll
      for (int i = 0; i < kNV; ++i) h[i] = in.get(1, i);
      if (a.post_norm) {
        const float2 st = row_stats<kNV>(h, last, a.post_norm, a.eps, inv_w, sum);
        const f32x2 r = splat2(st.y), m = splat2(-st.x * st.y);
#pragma unroll
        for (int i = 0; i < kNV; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) h[i].p[e] = fma_f32x2(h[i].p[e], r, m);
      }
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) t[i].p[e] = fma_f32x2(gate[i].p[e], h[i].p[e], t[i].p[e]);
        if (a.x_out && (i < kNV - 1 || last)) *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(a.x_out) + off + i * kVec) = pack_pairs(t[i]);
      }
    }
    in.next();
    in.load(src, off + (kNormFwdSlots - 1) * row_bytes, row + kNormFwdSlots - 1 < r1);
    if (!a.y) continue;
    const float2 st = a.norm ? row_stats<kNV>(t, last, a.norm, a.eps, inv_w, sum) : make_float2(0.f, 1.f);
    const f32x2 r = splat2(st.y), m = splat2(-st.x * st.y);
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      Pair8 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y.p[e] = fma_f32x2(fma_f32x2(t[i].p[e], r, m), scale[i].p[e], shift[i].p[e]);
      if (i < kNV - 1 || last) *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(a.y) + off + i * kVec) = pack_pairs(y);
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
// for the registers' sake; two blocks of 256 threads then share an SM.  Bound by the
// latency of a row's four exchanges and by issue (46 % of the slots): 5888 rows of 4096
// columns in two requests, both norms: 58 us, 5.0 TB/s, and the sums 6.  (A vector a thread and 512 threads
// at 64 registers spill: 183 us.)
template <int kNV, int kThreads>
__global__ void __launch_bounds__(kThreads, 512 / kThreads) gated_norm_backward_kernel(const __grid_constant__ NormSegs segs,
                                                                                      const __grid_constant__ NormArgs a) {
  extern __shared__ __align__(16) uint8_t smem_norm[];
  __shared__ float4 slots[2 * kThreads / 32];
  const int tid = threadIdx.x;
  const bool last = (tid + (kNV - 1) * kThreads) * 8 < a.width;
  const bool f32 = a.mod_f32 != 0;
  const int r0 = blockIdx.x * a.rows_per_block, r1 = r0 + min(a.rows - r0, a.rows_per_block);  // (the sum of the two may pass 2^31)
  const float inv_w = 1.f / static_cast<float>(a.width);
  BlockSum<kThreads / 32> sum{slots};
  constexpr uint32_t kVec = 16u * kThreads;  // bytes between a thread's vectors
  const int64_t row_bytes = 2 * static_cast<int64_t>(a.width);
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  const uint16_t* const src[4] = {a.dy ? a.x : nullptr, a.branch, a.dy, a.dx_out};
  RowsAhead<kNV, kThreads, 4, kNormBwdSlots> in;
  in.init(smem_norm, src, last);
  int64_t off = r0 * row_bytes + 16 * tid;  // of this thread's first vector of the row
#pragma unroll
  for (int i = 0; i < kNormBwdSlots - 1; ++i) in.load(src, off + i * row_bytes, r0 + i < r1);
  // [scale or gate][vector][half][thread] float4
  float4* vecs = reinterpret_cast<float4*>(smem_norm + kNormBwdSlots * in.kSlot) + tid;
  auto vec = [&](int k, int i, int h) -> float4& { return vecs[((k * kNV + i) * 2 + h) * kThreads]; };
  auto get_vec = [&](int k, int i) -> Pair8 {
    const float4 p = vec(k, i, 0), q = vec(k, i, 1);
    return Pair8{{make_f32x2(p.x, p.y), make_f32x2(p.z, p.w), make_f32x2(q.x, q.y), make_f32x2(q.z, q.w)}};
  };
  Pair8 sa[kNV], sb[kNV], sg[kNV];
#pragma unroll
  for (int i = 0; i < kNV; ++i) sa[i] = sb[i] = sg[i] = pairs_of(fill8(0.f));
  int seg = segment_of(segs, r0) - 1, end = r0;
  const int kind = a.dy ? a.norm : kNormNone, post = a.branch ? a.post_norm : kNormNone;
#pragma unroll 1
  for (int row = r0; row < r1; ++row, off += row_bytes) {
    if (row >= end) {
      do end = segs.cu[++seg + 1];
      while (row >= end);  // (skips requests without rows)
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        float p[8], q[8];
        const bool on = i < kNV - 1 || last;
        const int col = 8 * (tid + i * kThreads);
        const Vec8 w = on && a.weight ? load_param8(a.weight, col, f32) : fill8(1.f);
        const Vec8 sc = on && a.scale ? load_param8(a.scale, seg * a.ld_scale + col, f32) : fill8(0.f);
        const Vec8 g = on && a.gate ? load_param8(a.gate, seg * a.ld_gate + col, f32) : fill8(1.f);
        const Vec8 pw = on && a.post_weight ? load_param8(a.post_weight, col, f32) : fill8(1.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = on ? fmaf(w.v[e], sc.v[e], w.v[e]) : 0.f;
          q[e] = on ? g.v[e] * pw.v[e] : 0.f;
        }
        vec(0, i, 0) = make_float4(p[0], p[1], p[2], p[3]);
        vec(0, i, 1) = make_float4(p[4], p[5], p[6], p[7]);
        vec(1, i, 0) = make_float4(q[0], q[1], q[2], q[3]);
        vec(1, i, 1) = make_float4(q[4], q[5], q[6], q[7]);
      }
    }
    in.load(src, off + (kNormBwdSlots - 1) * row_bytes, row + kNormBwdSlots - 1 < r1);
    asm volatile("cp.async.wait_group %0;" ::"n"(kNormBwdSlots - 1) : "memory");
    Pair8 x[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) x[i] = in.get(0, i);
    // statistics of both norms in the same exchanges
    float2 xs = make_float2(0.f, 1.f), fs = make_float2(0.f, 1.f);
    if (kind || post) {
      Pair8 f[kNV];  // (read again where it is used: for the registers' sake)
#pragma unroll
      for (int i = 0; i < kNV; ++i) f[i] = in.get(1, i);
      if (kind == kNormLayer || post == kNormLayer) {
        float m[2] = {sum_of<kNV>(x), sum_of<kNV>(f)};
        sum(m);
        if (kind == kNormLayer) xs.x = m[0] * inv_w;
        if (post == kNormLayer) fs.x = m[1] * inv_w;
      }
      float q[2] = {centered_squares<kNV>(x, xs.x, last), centered_squares<kNV>(f, fs.x, last)};
      sum(q);
      if (kind) xs.y = rsqrtf(q[0] * inv_w + a.eps);
      if (post) fs.y = rsqrtf(q[1] * inv_w + a.eps);
    }
    f32x2 u0 = splat2(0.f), u1 = splat2(0.f);
    const f32x2 xm = splat2(-xs.x * xs.y), xr = splat2(xs.y), fm = splat2(-fs.x * fs.y), fr = splat2(fs.y);
    Pair8 d[kNV];  // u, then d, then dh times post_weight
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      const Pair8 dy = in.get(2, i), w = get_vec(0, i);  // (zeros without dy)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[i].p[e] = fma_f32x2(x[i].p[e], xr, xm);
        sa[i].p[e] = add_f32x2(sa[i].p[e], dy.p[e]);
        sb[i].p[e] = fma_f32x2(dy.p[e], x[i].p[e], sb[i].p[e]);
        d[i].p[e] = mul_f32x2(dy.p[e], w.p[e]);
        u0 = add_f32x2(u0, d[i].p[e]);
        u1 = fma_f32x2(d[i].p[e], x[i].p[e], u1);
      }
    }
    float u2[2] = {sum2(u0), sum2(u1)};
    if (kind) sum(u2);
    const f32x2 mu = splat2(kind == kNormLayer ? -u2[0] * inv_w : 0.f), mux = splat2(kind ? -u2[1] * inv_w : 0.f);
    f32x2 d0 = splat2(0.f), d1 = splat2(0.f);
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      const Pair8 dxo = in.get(3, i);
#pragma unroll
      for (int e = 0; e < 4; ++e) d[i].p[e] = fma_f32x2(xr, add_f32x2(d[i].p[e], fma_f32x2(x[i].p[e], mux, mu)), dxo.p[e]);
      if (a.dx && (i < kNV - 1 || last)) *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(a.dx) + off + i * kVec) = pack_pairs(d[i]);
      if (!a.branch) continue;
      const Pair8 g = get_vec(1, i), f = in.get(1, i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x2 fhat = x[i].p[e] = fma_f32x2(f.p[e], fr, fm);  // (in x's place from here on)
        sg[i].p[e] = fma_f32x2(d[i].p[e], fhat, sg[i].p[e]);
        d[i].p[e] = mul_f32x2(d[i].p[e], g.p[e]);
        d0 = add_f32x2(d0, d[i].p[e]);
        d1 = fma_f32x2(d[i].p[e], fhat, d1);
      }
    }
    if (a.branch && a.d_branch) {
      float d2[2] = {sum2(d0), sum2(d1)};
      if (post) sum(d2);
      const f32x2 md = splat2(post == kNormLayer ? -d2[0] * inv_w : 0.f), mdf = splat2(post ? -d2[1] * inv_w : 0.f);
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) d[i].p[e] = mul_f32x2(fr, add_f32x2(d[i].p[e], fma_f32x2(x[i].p[e], mdf, md)));
        if (i < kNV - 1 || last) *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(a.d_branch) + off + i * kVec) = pack_pairs(d[i]);
      }
    }
    in.next();
    if (row + 1 == r1 || row + 1 == end) {
      float* p = a.part + static_cast<int64_t>(blockIdx.x + seg) * 3 * a.width + 8 * tid;
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        auto put = [&](int k, Pair8& s) {
          if (i < kNV - 1 || last) {
            float4 q[2];
            split_f32x2(s.p[0], q[0].x, q[0].y), split_f32x2(s.p[1], q[0].z, q[0].w);
            split_f32x2(s.p[2], q[1].x, q[1].y), split_f32x2(s.p[3], q[1].z, q[1].w);
            float4* to = reinterpret_cast<float4*>(p + static_cast<int64_t>(k) * a.width + 8 * i * kThreads);
            to[0] = q[0];
            to[1] = q[1];
          }
          s = pairs_of(fill8(0.f));
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

// The result of one request and column: sum k (A, B, G) is v.  Returns what it adds to the
// weight's gradient: nothing for a request without rows, whatever its gate and scale hold.
__device__ __forceinline__ float norm_param_grad(const NormSumArgs& a, int k, int s, int col, bool rows, float v) {
  const int64_t at = static_cast<int64_t>(s) * a.width + col;
  const bool f32 = a.mod_f32 != 0;
  if (!rows) {
    float* to = k == 0 ? a.d_shift : k == 1 ? a.d_scale : a.d_gate;
    if (to) to[at] = 0.f;
    return 0.f;
  }
  if (k == 0) {
    if (a.d_shift) a.d_shift[at] = v;
    return 0.f;
  }
  if (k == 1) {
    if (a.d_scale) a.d_scale[at] = a.weight ? v * load_param(a.weight, col, f32) : v;
    return (a.scale ? 1.f + load_param(a.scale, s * a.ld_scale + col, f32) : 1.f) * v;
  }
  if (a.d_gate) a.d_gate[at] = a.post_weight ? v * load_param(a.post_weight, col, f32) : v;
  return (a.gate ? load_param(a.gate, s * a.ld_gate + col, f32) : 1.f) * v;
}
__device__ __forceinline__ void norm_weight_grad(const NormSumArgs& a, int k, int col, float total) {
  float* w = k == 1 ? a.d_weight : k == 2 ? a.d_post_weight : nullptr;
  if (w) w[col] = a.add ? w[col] + total : total;
}

// The parameters' gradients from the blocks' sums, which are read once; blockIdx.y = which
// sum.  One request, or some, for each blockIdx.z, or all of them one after the other where a
// weight's gradient needs their sum (gridDim.z = 1).  Two forms, for many and for few slots a
// request; all orders are fixed.
//
// Many: kSumCols columns a block, four for each of kSumCols / 4 threads that take every
// kSumGroups-th slot, so that most of its loads are under way at once; a warp's groups are
// joined by shuffles and the warps in their order.  295 slots of 4096 columns (14.7 MB) add
// 6 us to the call that wrote them.
constexpr int kSumThreads = 512, kSumWarps = kSumThreads / 32, kSumCols = 32, kSumGroups = kSumThreads / (kSumCols / 4);
__global__ void __launch_bounds__(kSumThreads) norm_param_grad_kernel(const __grid_constant__ NormSegs segs,
                                                                      const __grid_constant__ NormSumArgs a) {
  __shared__ float4 sums[kSumWarps][kSumCols / 4];
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  const int tid = threadIdx.x, k = blockIdx.y, g = tid / (kSumCols / 4), first = kSumCols * blockIdx.x;
  const int col = first + 4 * (tid % (kSumCols / 4)), mine = first + tid;  // of the loads; of the results (the first warp)
  const bool all = gridDim.z == 1;
  const int s1 = all ? segs.n : static_cast<int>(blockIdx.z) + 1;
  float total = 0.f;
  for (int s = all ? 0 : blockIdx.z; s < s1; ++s) {
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (col < a.width && segs.cu[s + 1] > segs.cu[s]) {
      const int b0 = segs.cu[s] / a.rows_per_block, b1 = (segs.cu[s + 1] - 1) / a.rows_per_block;
      const float* p = a.part + (static_cast<int64_t>(s) * 3 + k) * a.width + col;
#pragma unroll 4
      for (int b = b0 + g; b <= b1; b += kSumGroups) {
        const float4 v = *reinterpret_cast<const float4*>(p + static_cast<int64_t>(b) * 3 * a.width);
        sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
      }
    }
#pragma unroll
    for (int o = kSumCols / 4; o < 32; o <<= 1) {
      sum.x += __shfl_xor_sync(0xffffffffu, sum.x, o);
      sum.y += __shfl_xor_sync(0xffffffffu, sum.y, o);
      sum.z += __shfl_xor_sync(0xffffffffu, sum.z, o);
      sum.w += __shfl_xor_sync(0xffffffffu, sum.w, o);
    }
    if ((tid & 31) < kSumCols / 4) sums[tid >> 5][tid & 31] = sum;
    __syncthreads();
    if (tid < kSumCols && mine < a.width) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kSumWarps; ++w) v += reinterpret_cast<const float*>(sums[w])[tid];
      total += norm_param_grad(a, k, s, mine, segs.cu[s + 1] > segs.cu[s], v);
    }
    __syncthreads();
  }
  if (tid < kSumCols && mine < a.width) norm_weight_grad(a, k, mine, total);
}

// Few: 128 columns a block, four a lane, and a request for each warp.
constexpr int kSumFewCols = 128;
__global__ void __launch_bounds__(kSumThreads) norm_param_grad_few_kernel(const __grid_constant__ NormSegs segs,
                                                                          const __grid_constant__ NormSumArgs a) {
  __shared__ float4 sums[kSumWarps][32];
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.y, col = kSumFewCols * blockIdx.x + 4 * lane;
  const bool on = col < a.width;
  float4 total = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = kSumWarps * blockIdx.z + warp; on && s < segs.n; s += kSumWarps * gridDim.z) {
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    const bool rows = segs.cu[s + 1] > segs.cu[s];
    if (rows) {
      const int b0 = segs.cu[s] / a.rows_per_block, b1 = (segs.cu[s + 1] - 1) / a.rows_per_block;
      const float* p = a.part + (static_cast<int64_t>(s) * 3 + k) * a.width + col;
#pragma unroll 4
      for (int b = b0; b <= b1; ++b) {
        const float4 v = *reinterpret_cast<const float4*>(p + static_cast<int64_t>(b) * 3 * a.width);
        sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
      }
    }
    total.x += norm_param_grad(a, k, s, col, rows, sum.x);
    total.y += norm_param_grad(a, k, s, col + 1, rows, sum.y);
    total.z += norm_param_grad(a, k, s, col + 2, rows, sum.z);
    total.w += norm_param_grad(a, k, s, col + 3, rows, sum.w);
  }
  sums[warp][lane] = total;
  __syncthreads();
  const int mine = kSumFewCols * blockIdx.x + threadIdx.x;
  if (gridDim.z > 1 || threadIdx.x >= kSumFewCols || mine >= a.width) return;
  float v = 0.f;
#pragma unroll
  for (int w = 0; w < kSumWarps; ++w) v += reinterpret_cast<const float*>(sums[w])[threadIdx.x];
  norm_weight_grad(a, k, mine, v);
}

}  // namespace rc
