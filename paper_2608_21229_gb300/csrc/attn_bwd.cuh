// attn_bwd.cuh -- the gradients of the joint attention: what the backward kernels
// share (work description, the pass over the outputs), and the kernels on the
// legacy mma.sync path.
//
// With P = exp(scale Q K^T - lse), recomputed from the forward call's log-sum-exp,
//   dV = P^T dO,   dP = dO V^T,   dS = P (dP - delta),   delta = sum over d of dO O,
//   dQ = scale dS K,   dK = scale dS^T Q
// over the visible (query, key) pairs of one head: rows of a request see key range
// A and key range B (common.cuh), so the queries that see a key are one run of rows.
//
// Two kernels, each with its sums in one place: dK and dV of a key tile from all
// its queries, dQ of a query tile from all its keys.  Each computes S and dP for
// itself (7 products per pair of tiles, where one kernel with dQ added up in
// memory would take 5), and in return no sum crosses CTAs: no atomics, no fp32
// image of dQ in memory, and the same inputs give the same bits, as the forward
// calls promise.
//
// Scores, dP, P and dS are fp32 and so are all sums.  P and dS are rounded to bf16 where
// they become operands: a 16-bit MMA takes both of its operands in one type, and the
// other one here (dO, Q or K) is bf16; in TF32 three of the seven products would run at half
// the rate on operands of twice the size.  The gradients are then 0.0024 to 0.0026 from
// those in 64 bits (relative 2-norm), where their own rounding to bf16 alone makes 0.0017 to 0.0019.
//
// The cached rows' gradients (kRef32) may also be fp32: what steps add to from call to call
// then is not rounded to bf16 each time.  1280 queries, 3328 keys, 24 heads of 128: 120.6
// us written in bf16 and 128.6 added, 127.5 and 142.4 in fp32.
#pragma once
#include <cuda_bf16.h>

#include <type_traits>

#include "attn_mma.cuh"
#include "common.cuh"
#include "vec8.cuh"

namespace rc {

constexpr int kBwdMaxSegs = 64;

// A run of query rows that see key rows [a_row0, a_row0 + a_len) of the call's
// keys and [b_row0, b_row0 + b_len) of the cache.
struct BwdQuerySeg {
  int32_t q_row0, q_rows, a_row0, a_len, b_row0, b_len;
  int32_t tile0;  // first query tile of the launch
};
// A run of key rows (of the call's keys, or of the cache) that all of query rows
// [q_row0, q_row0 + q_rows) see.  Row k_row0 + i with i >= add_from has the
// gradient in row add_row0 + i of the tensors `add` added to its own.
struct BwdKeySeg {
  int32_t k_row0, k_rows, q_row0, q_rows;
  int32_t in_b, add_from, add_row0;
  int32_t tile0;
};
struct BwdQueries {
  BwdQuerySeg seg[kBwdMaxSegs];
  int32_t n, n_tiles;
};
struct BwdKeys {
  BwdKeySeg seg[kBwdMaxSegs];
  int32_t n, n_tiles;
};

struct BwdArgs {
  const __nv_bfloat16 *q, *ka, *va, *kb, *vb, *d_o;
  __nv_bfloat16 *dq, *dka, *dva;
  void *dkb, *dvb;            // gradients of the cached rows, bf16 or (kRef32 kernels) fp32
  const void *add_k, *add_v;  // see BwdKeySeg; of the same type
  const float2* stats;                 // [heads][rows]: (lse log2 e, delta) of each query row
  int64_t row_stride;                  // elements between rows (= H * D)
  int64_t rows;                        // query rows
  int64_t a_rows, b_rows;              // rows of the call's key tensors and of the cache's
  int32_t num_heads;
  float scale, scale_log2;
  uint64_t timeout_ns;
  int* status;
  int *work_keys, *work_queries;  // tcgen05 kernels: counters of items, zero at launch (null: fixed order)
  int32_t behind_queries;         // keys kernel: launched right behind the queries kernel
  int32_t dbg_stop;               // tcgen05 kernels: refcache_debug_skip_first_load's argument
  uint64_t* passed;               // tcgen05 kernels: see kBwdPassed
  uint64_t ticket;
};
// The workspace of a call: the statistics, then words that the pass over the outputs sets to
// zero: a pair of counters for each list of requests, and in the last two the ticket with
// which the queries kernel says that it has passed its wait for that pass.  The keys kernel
// starts while the queries kernel runs, and griddepcontrol.wait would hold it until that has
// ended; a ticket read with acquire orders it behind the release in the queries kernel, and
// so behind all that this one's wait has made visible.  The ticket is the call's own (a random
// sequence of 64 bits) and the keys kernel sets the word back to zero at its end, so that a
// replayed graph never finds that of the replay before.  No ticket there: the keys kernel
// waits in the ordinary way.
constexpr int kBwdCounters = 256, kBwdPassed = kBwdCounters - 2;

// Item `it` of a list: runs in the list's order (longest first), within a run
// head by head, so that the CTAs that work at the same time share few heads' rows
// in the L2.
struct BwdItem {
  int seg, head, tile;  // tile within the run
};
template <typename List>
__device__ __forceinline__ BwdItem bwd_item(const List& l, int it, int num_heads) {
  const int at = it / num_heads;
  int lo = 0, hi = l.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (l.seg[mid].tile0 <= at)
      lo = mid;
    else
      hi = mid - 1;
  }
  const int first = l.seg[lo].tile0, tiles = (lo + 1 < l.n ? l.seg[lo + 1].tile0 : l.n_tiles) - first;
  const int r = it - first * num_heads;
  return BwdItem{lo, r / tiles, r % tiles};
}

// stats[head][row] = (lse log2 e, delta).  A block takes 256 / (D / 8) rows of four
// heads; bound by reading dO and O once (the statistics lie by head, as the kernels read
// them, so four heads a block: 128 bytes of lse and of statistics a line).  1280 rows of 24
// heads of 128 take 6.0 us (15.9 MB), 9431 rows of 16 heads of 64 11 us (39 MB, 3.6 TB/s).
constexpr int kBwdPrepHeads = 4;
template <int D>
__global__ void __launch_bounds__(256) attn_bwd_prep_kernel(const __nv_bfloat16* o, const __nv_bfloat16* d_o, const float* lse,
                                                            float2* stats, int64_t rows, int num_heads) {
  constexpr int kLanes = D / 8, kRows = 256 / kLanes;
  grid_dependency_wait();
  if (threadIdx.x == 0) grid_launch_dependents();
  static_assert(kBwdCounters == 256, "one counter per thread");
  if (blockIdx.x == 0 && blockIdx.y == 0) reinterpret_cast<int*>(stats + rows * num_heads)[threadIdx.x] = 0;
  const int l = threadIdx.x % kLanes;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kLanes;
  const int h0 = blockIdx.y * kBwdPrepHeads;
  const bool on = row < rows;
  uint4 a[kBwdPrepHeads], b[kBwdPrepHeads];
  float ls[kBwdPrepHeads];
#pragma unroll
  for (int i = 0; i < kBwdPrepHeads; ++i) {
    a[i] = b[i] = make_uint4(0, 0, 0, 0);
    ls[i] = 0.f;
    if (on && h0 + i < num_heads) {
      const int64_t at = (row * num_heads + h0 + i) * D + 8 * l;
      a[i] = *reinterpret_cast<const uint4*>(o + at);
      b[i] = *reinterpret_cast<const uint4*>(d_o + at);
      ls[i] = lse[row * num_heads + h0 + i];
    }
  }
#pragma unroll
  for (int i = 0; i < kBwdPrepHeads; ++i) {
    const Vec8 x = unpack8(a[i]), y = unpack8(b[i]);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x.v[e], y.v[e], s);
#pragma unroll
    for (int k = kLanes / 2; k > 0; k >>= 1) s += __shfl_xor_sync(0xffffffffu, s, k);
    if (l == 0 && on && h0 + i < num_heads)
      stats[static_cast<int64_t>(h0 + i) * rows + row] = make_float2(ls[i] * 1.4426950408889634f, s);
  }
}

// ---------------------------------------------------------------- mma.sync
// The plain form of the two kernels, kept beside the tcgen05 ones as attn_mma_kernel is
// beside the forward's: a second implementation that the tests compare.  Bound by the
// mma.sync pipe and its operands' way through registers: 4608 queries and 25088 keys of 24
// heads of 128 take 15.2 ms (234 TFLOP/s of the five products, 2.8 ms on tcgen05).
namespace mm {
constexpr int kBwdRows = 64;  // rows of a CTA (keys or queries), 16 per warp
constexpr int kBwdStep = 32;  // rows of the other side per step
template <int D>
constexpr int bwd_smem() {
  return (2 * kBwdRows + 4 * kBwdStep) * D * 2 + 2 * kBwdStep * 8;
}

// C[16 x 32] = A[16 x D] B[32 x D]^T, A in rows 16 warp.. of `a`, B rows of `b`, both in
// shared memory in 16-byte chunks swizzled by row.
template <int D, typename Off>
__device__ __forceinline__ void rows_by_rows(float (&c)[4][4], const __nv_bfloat16* a, const __nv_bfloat16* b, int warp, int mi,
                                             int li, const Off& off) {
#pragma unroll
  for (int n = 0; n < 4; ++n) c[n][0] = c[n][1] = c[n][2] = c[n][3] = 0.f;
#pragma unroll
  for (int kt = 0; kt < D / 16; ++kt) {
    uint32_t fa[4];
    ldsm_x4(fa, a + off(16 * warp + (mi & 1) * 8 + li, 2 * kt + (mi >> 1)));
#pragma unroll
    for (int np = 0; np < 2; ++np) {
      uint32_t fb[4];
      ldsm_x4(fb, b + off(16 * np + (mi >> 1) * 8 + li, 2 * kt + (mi & 1)));
      mma16816(c[2 * np], fa, fb[0], fb[1]);
      mma16816(c[2 * np + 1], fa, fb[2], fb[3]);
    }
  }
}
// acc[16 x D] += W[16 x 32] B[32 x D], W as the accumulators of rows_by_rows rounded to bf16.
template <int D, typename Off>
__device__ __forceinline__ void add_weighted(float (&acc)[D / 8][4], const float (&w)[4][4], const __nv_bfloat16* b, int mi, int li,
                                             const Off& off) {
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    const uint32_t fa[4] = {pack2(w[2 * kt][0], w[2 * kt][1]), pack2(w[2 * kt][2], w[2 * kt][3]),
                            pack2(w[2 * kt + 1][0], w[2 * kt + 1][1]), pack2(w[2 * kt + 1][2], w[2 * kt + 1][3])};
#pragma unroll
    for (int dp = 0; dp < D / 16; ++dp) {
      uint32_t fb[4];
      ldsm_x4_t(fb, b + off(16 * kt + (mi & 1) * 8 + li, 2 * dp + (mi >> 1)));
      mma16816(acc[2 * dp], fa, fb[0], fb[1]);
      mma16816(acc[2 * dp + 1], fa, fb[2], fb[3]);
    }
  }
}
}  // namespace mm

// dK and dV of 64 keys (16 per warp): S^T = K Q^T and dP^T = V dO^T, 32 queries at a time.
// kRef32: the cached rows' gradients are fp32, here and in what is added.
template <int D, bool kRef32>
__global__ void __launch_bounds__(128) attn_bwd_mma_keys_kernel(const __grid_constant__ BwdKeys keys, const BwdArgs a) {
  using namespace mm;
  extern __shared__ __align__(128) uint8_t smem_mm[];
  __nv_bfloat16* sK = reinterpret_cast<__nv_bfloat16*>(smem_mm);
  __nv_bfloat16* sV = sK + kBwdRows * D;
  __nv_bfloat16* sQ = sV + kBwdRows * D;  // two buffers of Q rows, then two of dO rows
  __nv_bfloat16* sO = sQ + 2 * kBwdStep * D;
  float2* sT = reinterpret_cast<float2*>(sO + 2 * kBwdStep * D);
  auto off = [](int row, int ch) { return row * D + ((ch ^ (row & 7)) << 3); };
  const BwdItem item = bwd_item(keys, blockIdx.x, a.num_heads);
  const int head = item.head;
  const BwdKeySeg sg = keys.seg[item.seg];
  const int r0 = item.tile * kBwdRows, nk = min(kBwdRows, sg.k_rows - r0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t ld = a.row_stride;
  auto load_rows = [&](__nv_bfloat16* dst, const __nv_bfloat16* src, int64_t row0, int n, int valid) {
    for (int i = threadIdx.x; i < n * (D / 8); i += 128) {
      const int r = i / (D / 8), ch = i % (D / 8);
      cp_async16(dst + off(r, ch), src + (row0 + (r < valid ? r : 0)) * ld + head * D + ch * 8, r < valid ? 16 : 0);
    }
  };
  auto load_step = [&](int j) {
    const int64_t row0 = sg.q_row0 + kBwdStep * j;
    const int valid = min(kBwdStep, sg.q_rows - kBwdStep * j), b = j & 1;
    load_rows(sQ + b * kBwdStep * D, a.q, row0, kBwdStep, valid);
    load_rows(sO + b * kBwdStep * D, a.d_o, row0, kBwdStep, valid);
    if (threadIdx.x < kBwdStep)
      sT[b * kBwdStep + threadIdx.x] = static_cast<int>(threadIdx.x) < valid ? a.stats[head * a.rows + row0 + threadIdx.x]
                                                                             : make_float2(INFINITY, 0.f);
  };
  const int steps = (sg.q_rows + kBwdStep - 1) / kBwdStep;
  load_rows(sK, sg.in_b ? a.kb : a.ka, sg.k_row0 + r0, kBwdRows, nk);
  load_rows(sV, sg.in_b ? a.vb : a.va, sg.k_row0 + r0, kBwdRows, nk);
  if (steps > 0) load_step(0);
  cp_async_commit();
  const int g = lane >> 2, q4 = lane & 3, mi = lane >> 3, li = lane & 7;
  float dk[D / 8][4], dv[D / 8][4];
#pragma unroll
  for (int i = 0; i < D / 8; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) dk[i][e] = dv[i][e] = 0.f;
  for (int j = 0; j < steps; ++j) {
    const int b = j & 1;
    if (j + 1 < steps) {
      load_step(j + 1);
      cp_async_commit();
      cp_async_wait<1>();
    } else {
      cp_async_wait<0>();
    }
    __syncthreads();
    const __nv_bfloat16 *Q = sQ + b * kBwdStep * D, *O = sO + b * kBwdStep * D;
    const float2* T = sT + b * kBwdStep;
    float p[4][4], ds[4][4];
    rows_by_rows<D>(p, sK, Q, warp, mi, li, off);
    rows_by_rows<D>(ds, sV, O, warp, mi, li, off);
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 t = T[8 * n + 2 * q4 + (e & 1)];
        p[n][e] = ex2f(fmaf(p[n][e], a.scale_log2, -t.x));
        ds[n][e] = p[n][e] * (ds[n][e] - t.y);
      }
    add_weighted<D>(dv, p, O, mi, li, off);
    add_weighted<D>(dk, ds, Q, mi, li, off);
    __syncthreads();
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = r0 + 16 * warp + g + 8 * h;
    if (r >= sg.k_rows) continue;
    const int64_t at = (sg.k_row0 + r) * ld + head * D;
    const bool add = r >= sg.add_from;
    const int64_t from = (static_cast<int64_t>(sg.add_row0) + r) * ld + head * D;
    using Ref = std::conditional_t<kRef32, float, __nv_bfloat16>;
    uint32_t* ok = reinterpret_cast<uint32_t*>((sg.in_b ? static_cast<__nv_bfloat16*>(a.dkb) : a.dka) + at);
    uint32_t* ov = reinterpret_cast<uint32_t*>((sg.in_b ? static_cast<__nv_bfloat16*>(a.dvb) : a.dva) + at);
    const Ref *add_k = static_cast<const Ref*>(a.add_k) + from, *add_v = static_cast<const Ref*>(a.add_v) + from;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const int c = 4 * i + q4;
      float k0 = dk[i][2 * h] * a.scale, k1 = dk[i][2 * h + 1] * a.scale, v0 = dv[i][2 * h], v1 = dv[i][2 * h + 1];
      if (add) {
        if constexpr (kRef32) {
          const float2 xk = reinterpret_cast<const float2*>(add_k)[c], xv = reinterpret_cast<const float2*>(add_v)[c];
          k0 += xk.x, k1 += xk.y, v0 += xv.x, v1 += xv.y;
        } else {
          const uint32_t xk = reinterpret_cast<const uint32_t*>(add_k)[c], xv = reinterpret_cast<const uint32_t*>(add_v)[c];
          k0 += __uint_as_float(xk << 16), k1 += __uint_as_float(xk & 0xFFFF0000u);
          v0 += __uint_as_float(xv << 16), v1 += __uint_as_float(xv & 0xFFFF0000u);
        }
      }
      if (kRef32 && sg.in_b) {
        reinterpret_cast<float2*>(static_cast<float*>(a.dkb) + at)[c] = make_float2(k0, k1);
        reinterpret_cast<float2*>(static_cast<float*>(a.dvb) + at)[c] = make_float2(v0, v1);
        continue;
      }
      ok[c] = pack2(k0, k1);
      ov[c] = pack2(v0, v1);
    }
  }
}

// dQ of 64 queries (16 per warp): S = Q K^T and dP = dO V^T, 32 keys at a time.
template <int D>
__global__ void __launch_bounds__(128) attn_bwd_mma_queries_kernel(const __grid_constant__ BwdQueries queries, const BwdArgs a) {
  using namespace mm;
  extern __shared__ __align__(128) uint8_t smem_mm[];
  __nv_bfloat16* sQ = reinterpret_cast<__nv_bfloat16*>(smem_mm);
  __nv_bfloat16* sO = sQ + kBwdRows * D;
  __nv_bfloat16* sK = sO + kBwdRows * D;
  __nv_bfloat16* sV = sK + 2 * kBwdStep * D;
  auto off = [](int row, int ch) { return row * D + ((ch ^ (row & 7)) << 3); };
  const BwdItem item = bwd_item(queries, blockIdx.x, a.num_heads);
  const int head = item.head;
  const BwdQuerySeg sg = queries.seg[item.seg];
  const int r0 = item.tile * kBwdRows, nq = min(kBwdRows, sg.q_rows - r0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t ld = a.row_stride;
  auto load_rows = [&](__nv_bfloat16* dst, const __nv_bfloat16* src, int64_t row0, int n, int valid) {
    for (int i = threadIdx.x; i < n * (D / 8); i += 128) {
      const int r = i / (D / 8), ch = i % (D / 8);
      cp_async16(dst + off(r, ch), src + (row0 + (r < valid ? r : 0)) * ld + head * D + ch * 8, r < valid ? 16 : 0);
    }
  };
  const int na = (sg.a_len + kBwdStep - 1) / kBwdStep, steps = na + (sg.b_len + kBwdStep - 1) / kBwdStep;
  auto valid_of = [&](int j) { return j < na ? min(kBwdStep, sg.a_len - kBwdStep * j) : min(kBwdStep, sg.b_len - kBwdStep * (j - na)); };
  auto load_step = [&](int j) {
    const int64_t row0 = j < na ? sg.a_row0 + kBwdStep * j : sg.b_row0 + kBwdStep * (j - na);
    const int b = j & 1;
    load_rows(sK + b * kBwdStep * D, j < na ? a.ka : a.kb, row0, kBwdStep, valid_of(j));
    load_rows(sV + b * kBwdStep * D, j < na ? a.va : a.vb, row0, kBwdStep, valid_of(j));
  };
  load_rows(sQ, a.q, sg.q_row0 + r0, kBwdRows, nq);
  load_rows(sO, a.d_o, sg.q_row0 + r0, kBwdRows, nq);
  if (steps > 0) load_step(0);
  cp_async_commit();
  const int g = lane >> 2, q4 = lane & 3, mi = lane >> 3, li = lane & 7;
  float2 t[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = 16 * warp + g + 8 * h;
    t[h] = r < nq ? a.stats[head * a.rows + sg.q_row0 + r0 + r] : make_float2(INFINITY, 0.f);
  }
  float dq[D / 8][4];
#pragma unroll
  for (int i = 0; i < D / 8; ++i) dq[i][0] = dq[i][1] = dq[i][2] = dq[i][3] = 0.f;
  for (int j = 0; j < steps; ++j) {
    const int b = j & 1, valid = valid_of(j);
    if (j + 1 < steps) {
      load_step(j + 1);
      cp_async_commit();
      cp_async_wait<1>();
    } else {
      cp_async_wait<0>();
    }
    __syncthreads();
    float p[4][4], ds[4][4];
    rows_by_rows<D>(p, sQ, sK + b * kBwdStep * D, warp, mi, li, off);
    rows_by_rows<D>(ds, sO, sV + b * kBwdStep * D, warp, mi, li, off);
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 r = t[e >> 1];
        const float w = 8 * n + 2 * q4 + (e & 1) < valid ? ex2f(fmaf(p[n][e], a.scale_log2, -r.x)) : 0.f;
        ds[n][e] = w * (ds[n][e] - r.y);
      }
    add_weighted<D>(dq, ds, sK + b * kBwdStep * D, mi, li, off);
    __syncthreads();
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = 16 * warp + g + 8 * h;
    if (r >= nq) continue;
    uint32_t* dst = reinterpret_cast<uint32_t*>(a.dq + (sg.q_row0 + r0 + r) * ld + head * D);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) dst[4 * i + q4] = pack2(dq[i][2 * h] * a.scale, dq[i][2 * h + 1] * a.scale);
  }
}

}  // namespace rc
