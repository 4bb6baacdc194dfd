// block_ops.cu -- the entry points of include/refcache.h for what lies around the
// joint attention in a transformer block: projections to attention inputs
// (qkv_rope.cuh), gated norms (gated_norm.cuh) and the clipping of gradients
// (clip_grads.cuh).  Argument checks and launches; no call allocates memory.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <type_traits>

#include "refcache.h"
#include "clip_grads.cuh"
#include "gated_norm.cuh"
#include "host_common.h"
#include "qkv_rope.cuh"

using rc_host::aligned16;
using rc_host::cuda_fail;
using rc_host::device_sms;
using rc_host::fail;
using rc_host::launch_dependent;

namespace {

constexpr int64_t kMaxRows = (1ll << 31) - 1 - 512;
constexpr int kRopeMaxParts = 1024;   // blocks of the rotary gradient's launch
constexpr int kNormMaxBlocks = 1280;  // blocks of a gated norm's gradient launch
constexpr int kClipMaxBlocks = 2560;  // blocks of a norm launch of clip_gradients

int ceil_div(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }

int check_tensor(const void* p, const char* name) {
  if (!p) return fail(REFCACHE_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned16(p)) return fail(REFCACHE_ERR_INVALID_ARG, "%s: tensor pointer not 16-byte aligned", name);
  return REFCACHE_OK;
}
int check_optional(const void* p, const char* name) { return p ? check_tensor(p, name) : REFCACHE_OK; }
// fp32 results, each of which may be absent
int check_floats(std::initializer_list<const float*> tensors, const char* name) {
  for (const float* p : tensors)
    if (reinterpret_cast<uintptr_t>(p) & 3u) return fail(REFCACHE_ERR_INVALID_ARG, "%s: a float32 result is not 4-byte aligned", name);
  return REFCACHE_OK;
}

// ---------------------------------------------------------------- rotary positions
int check_rope(const refcache_rope_t* r, const refcache_rope_rows_t* w) {
  if (!r || !w) return fail(REFCACHE_ERR_INVALID_ARG, "qkv_rope: NULL rope or rows");
  if (r->head_dim != 64 && r->head_dim != 128)
    return fail(REFCACHE_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", r->head_dim);
  if (r->num_axes < 1 || r->num_axes > REFCACHE_ROPE_MAX_AXES)
    return fail(REFCACHE_ERR_INVALID_ARG, "qkv_rope: the rope was not made by refcache_rope_init");
  for (int j = 0; j < r->head_dim / 2; ++j)
    if (r->axis[j] >= r->num_axes) return fail(REFCACHE_ERR_INVALID_ARG, "qkv_rope: pair %d on axis %d of %d", j, r->axis[j], r->num_axes);
  if (w->num_heads < 1 || static_cast<int64_t>(w->num_heads) * r->head_dim > (1 << 20))
    return fail(REFCACHE_ERR_INVALID_ARG, "num_heads must be >= 1 and num_heads x head_dim at most 2^20 (got %d heads)", w->num_heads);
  if (w->rows < 0 || w->rows > kMaxRows || w->out_rows < 0 || w->out_rows > kMaxRows)
    return fail(REFCACHE_ERR_INVALID_ARG, "qkv_rope: rows outside [0, 2^31 - 513]");
  if (!w->row_map && w->out_rows < w->rows)
    return fail(REFCACHE_ERR_INVALID_ARG, "qkv_rope: %lld rows do not fit %lld rows of the outputs", static_cast<long long>(w->rows),
                static_cast<long long>(w->out_rows));
  if (!(w->eps >= 0.f) || !std::isfinite(w->eps)) return fail(REFCACHE_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (w->rows == 0) return REFCACHE_OK;
  if (!w->positions || (reinterpret_cast<uintptr_t>(w->positions) & 3u))
    return fail(REFCACHE_ERR_INVALID_ARG, "qkv_rope: positions is NULL or not 4-byte aligned");
  if (reinterpret_cast<uintptr_t>(w->row_map) & 3u) return fail(REFCACHE_ERR_INVALID_ARG, "qkv_rope: row_map not 4-byte aligned");
  int rc;
  if ((rc = check_optional(w->weight_q, "weight_q")) != 0) return rc;
  return check_optional(w->weight_k, "weight_k");
}

int check_ld(int64_t ld, int64_t least, const char* name) {
  if (ld < least || ld % 8)
    return fail(REFCACHE_ERR_INVALID_ARG, "%s: %lld elements between rows (a multiple of 8, at least %lld)", name,
                static_cast<long long>(ld), static_cast<long long>(least));
  return REFCACHE_OK;
}

void rope_tables(const refcache_rope_t* r, const refcache_rope_rows_t* w, rc::RopeTable* t, rc::RopeArgs* a) {
  for (int j = 0; j < rc::kRopeMaxPairs; ++j) {
    t->turn_hi[j] = r->turn_hi[j];
    t->turn_lo[j] = r->turn_lo[j];
    t->axis[j] = r->axis[j];
  }
  t->num_axes = r->num_axes;
  a->weight[0] = w->weight_q;
  a->weight[1] = w->weight_k;
  a->weight_f32 = w->weight_f32 != 0;
  a->positions = w->positions;
  a->row_map = w->row_map;
  a->rows = w->rows;
  a->out_rows = w->out_rows;
  a->num_heads = w->num_heads;
  a->eps = w->eps;
}

// Slices of the heads: few tokens leave SMs without a warp, so a token's heads are
// divided among up to as many warps as have a full set of loads each, as long as there are
// fewer than 56 an SM (32 are resident; 24 heads of 128, 2500 rows: one slice 22.5 us, three 18.3).
int rope_slices(const refcache_rope_t* r, const refcache_rope_rows_t* w, int sms, int unroll, int* step) {
  const int per = 32 / (r->head_dim / 8), most = std::min(64, ceil_div(w->num_heads, unroll * per));
  const int64_t want = 56ll * sms / w->rows;
  int slices = static_cast<int>(std::min<int64_t>(most, std::max<int64_t>(1, want)));
  *step = ceil_div(ceil_div(w->num_heads, slices), per) * per;
  return ceil_div(w->num_heads, *step);
}

// The gradient's blocks of each slice.  Every block stays for the whole launch, so the slices
// are as many as let the warp with the most rows have the fewest heads in all; a row's angles
// count as three.  24 heads of 128, one slice and as chosen: 2500 rows 37.5 and 32.0
// us (three), 20608 rows 177 and 204 with three.
int rope_backward_blocks(const refcache_rope_t* r, const refcache_rope_rows_t* w, int resident, int unroll, int* slices, int* step) {
  const int per = 32 / (r->head_dim / 8), most = std::min(64, ceil_div(w->num_heads, unroll * per));
  int64_t best = INT64_MAX;
  int blocks = 1;
  for (int want = 1; want <= most; ++want) {
    const int heads = ceil_div(ceil_div(w->num_heads, want), per) * per, n = ceil_div(w->num_heads, heads);
    const int b = std::min(ceil_div(w->rows, rc::kRopeTokens), std::max(1, resident / n));
    const int64_t cost = ceil_div(w->rows, static_cast<int64_t>(b) * rc::kRopeTokens) * (heads + 3ll);
    if (cost < best) best = cost, blocks = b, *slices = n, *step = heads;
  }
  return blocks;
}

// ---------------------------------------------------------------- gated norm
int check_norm(const refcache_gated_norm_t* p) {
  if (!p) return fail(REFCACHE_ERR_INVALID_ARG, "gated_norm: NULL parameters");
  if (p->batch < 1) return fail(REFCACHE_ERR_INVALID_ARG, "batch must be >= 1 (got %d)", p->batch);
  if (!p->cu_rows || p->cu_rows[0] != 0) return fail(REFCACHE_ERR_INVALID_ARG, "cu_rows is NULL or cu_rows[0] is not 0");
  for (int b = 0; b < p->batch; ++b)
    if (p->cu_rows[b + 1] < p->cu_rows[b]) return fail(REFCACHE_ERR_INVALID_ARG, "cu_rows must be non-decreasing (at %d)", b);
  if (p->cu_rows[p->batch] > kMaxRows) return fail(REFCACHE_ERR_INVALID_ARG, "cu_rows: too many rows");
  if (p->width < 8 || p->width % 8 || p->width > rc::kNormMaxWidth)
    return fail(REFCACHE_ERR_UNSUPPORTED, "width must be a multiple of 8 in [8, %d] (got %d)", rc::kNormMaxWidth, p->width);
  if (p->norm < REFCACHE_NORM_NONE || p->norm > REFCACHE_NORM_RMS || p->post_norm < REFCACHE_NORM_NONE || p->post_norm > REFCACHE_NORM_RMS)
    return fail(REFCACHE_ERR_INVALID_ARG, "unknown norm %d or post_norm %d", p->norm, p->post_norm);
  if (!(p->eps >= 0.f) || !std::isfinite(p->eps)) return fail(REFCACHE_ERR_INVALID_ARG, "eps must be finite and >= 0");
  const void* tensors[] = {p->gate, p->scale, p->shift, p->weight, p->post_weight};
  const char* names[] = {"gate", "scale", "shift", "weight", "post_weight"};
  const int64_t lds[] = {p->ld_gate, p->ld_scale, p->ld_shift};
  for (int i = 0; i < 5; ++i) {
    int rc = check_optional(tensors[i], names[i]);
    if (rc) return rc;
    if (i < 3 && tensors[i] && lds[i] != 0 && (rc = check_ld(lds[i], p->width, names[i])) != 0) return rc;  // (0: one row for all)
  }
  if (p->post_weight && p->post_norm == REFCACHE_NORM_NONE)
    return fail(REFCACHE_ERR_INVALID_ARG, "post_weight without post_norm");
  return REFCACHE_OK;
}

// Requests [b, b + n) as one launch: rows from cu_rows[b] on.
rc::NormSegs norm_segs(const refcache_gated_norm_t* p, int b, int n) {
  rc::NormSegs s{};
  s.n = n;
  for (int i = 0; i <= n; ++i) s.cu[i] = p->cu_rows[b + i] - p->cu_rows[b];
  return s;
}

const void* at_row(const void* p, int64_t elems, bool f32) {
  return p ? static_cast<const uint8_t*>(p) + elems * (f32 ? 4 : 2) : nullptr;
}

rc::NormArgs norm_args(const refcache_gated_norm_t* p, int b, int rows) {
  const bool f32 = p->mod_f32 != 0;
  rc::NormArgs a{};
  a.gate = at_row(p->gate, b * p->ld_gate, f32);
  a.scale = at_row(p->scale, b * p->ld_scale, f32);
  a.shift = at_row(p->shift, b * p->ld_shift, f32);
  a.weight = p->weight;
  a.post_weight = p->post_weight;
  a.ld_gate = p->ld_gate;
  a.ld_scale = p->ld_scale;
  a.ld_shift = p->ld_shift;
  a.rows = rows;
  a.width = p->width;
  a.norm = p->norm;
  a.post_norm = p->post_norm;
  a.mod_f32 = f32;
  a.eps = p->eps;
  return a;
}

// A block's threads for a row of `width` (a power of two, with one vector of the row each
// up to 2048 columns, two above) and its shared memory.
struct NormShape {
  int nv, threads, smem;
};
NormShape norm_shape(int width, bool backward) {
  const int nvec = width / 8;
  NormShape n{};
  n.nv = nvec <= 256 ? 1 : 2;
  n.threads = 32;
  while (n.threads * n.nv < nvec) n.threads *= 2;
  n.smem = n.nv * n.threads * 16 * (backward ? rc::kNormBwdSlots * 4 + 4 : rc::kNormFwdSlots * 2);
  return n;
}
// Blocks: as many as an SM holds (of 65536 registers, 128 a thread, and 227 KB), and at
// most a row each.
int norm_blocks(int rows, int sms, const NormShape& n) {
  const int per_sm = std::max(1, std::min({512 / n.threads, (227 << 10) / (n.smem + 2048), 16}));
  return std::min(rows, per_sm * sms);
}
// Rows of a forward block.  SMs run at different speeds, so more blocks than are resident at
// once end sooner, as long as a block has enough rows to be worth its start (16, or 32 where
// one block has an SM to itself): as many whole rounds of resident blocks as leave that.
// One round against these, no post norm and with one: 8704 rows of 4096 53.6 and 49.0 us
// (two rounds), 9216 rows 56.3 and 50.5, 52.2 and 53.5; 40000 rows of 2048 123 and 104, 164
// and 120 (eight); 20000 rows of 2048 with ten rows a block 53 and 65, with these 55 and 63.
int norm_rows_per_block(int rows, int sms, const NormShape& n) {
  const int64_t resident = norm_blocks(rows, sms, n), least = (n.threads < 512 ? 16 : 32) * resident;
  return ceil_div(rows, resident * std::max<int64_t>(1, (rows + least / 2) / least));
}
// f(kNV, kThreads) of the shape, as constants.
template <typename F>
cudaError_t with_norm_shape(const NormShape& n, const F& f) {
  using std::integral_constant;
  if (n.nv == 2)
    return n.threads == 256 ? f(integral_constant<int, 2>{}, integral_constant<int, 256>{})
                            : f(integral_constant<int, 2>{}, integral_constant<int, 512>{});
  switch (n.threads) {
    case 32: return f(integral_constant<int, 1>{}, integral_constant<int, 32>{});
    case 64: return f(integral_constant<int, 1>{}, integral_constant<int, 64>{});
    case 128: return f(integral_constant<int, 1>{}, integral_constant<int, 128>{});
    default: return f(integral_constant<int, 1>{}, integral_constant<int, 256>{});
  }
}
template <typename Kernel>
cudaError_t launch_norm(Kernel kernel, const NormShape& n, int blocks, cudaStream_t s, const rc::NormSegs& segs, const rc::NormArgs& a) {
  if (n.smem > 40 << 10) {  // (with the static part, above what a launch may have by default)
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, n.smem);
    if (e != cudaSuccess) return e;
  }
  return launch_dependent(kernel, dim3(static_cast<unsigned>(blocks)), dim3(static_cast<unsigned>(n.threads)), n.smem, s, segs, a);
}

}  // namespace

extern "C" {

int refcache_rope_init(refcache_rope_t* r, int head_dim, int num_axes, const int32_t* axis_dims, double theta, int interleaved) {
  if (!r || !axis_dims) return fail(REFCACHE_ERR_INVALID_ARG, "refcache_rope_init: NULL argument");
  if (head_dim != 64 && head_dim != 128) return fail(REFCACHE_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", head_dim);
  if (num_axes < 1 || num_axes > REFCACHE_ROPE_MAX_AXES)
    return fail(REFCACHE_ERR_INVALID_ARG, "num_axes must be in [1, %d] (got %d)", REFCACHE_ROPE_MAX_AXES, num_axes);
  if (!(theta > 0.0) || !std::isfinite(theta)) return fail(REFCACHE_ERR_INVALID_ARG, "theta must be finite and > 0");
  int64_t sum = 0;
  for (int i = 0; i < num_axes; ++i) {
    if (axis_dims[i] < 0 || axis_dims[i] % 2)
      return fail(REFCACHE_ERR_INVALID_ARG, "axis_dims[%d] = %d is negative or odd", i, axis_dims[i]);
    sum += axis_dims[i];
  }
  if (sum > head_dim) return fail(REFCACHE_ERR_INVALID_ARG, "the axes' dims add up to %lld, above head_dim %d", static_cast<long long>(sum), head_dim);
  *r = refcache_rope_t{};
  r->head_dim = head_dim;
  r->num_axes = num_axes;
  r->interleaved = interleaved != 0;
  int j = 0;
  for (int i = 0; i < num_axes; ++i)
    for (int k = 0; k < axis_dims[i] / 2; ++k, ++j) {
      const double turns = std::pow(theta, -2.0 * k / axis_dims[i]) / 6.283185307179586476925;
      r->turn_hi[j] = static_cast<float>(turns);
      r->turn_lo[j] = static_cast<float>(turns - static_cast<double>(r->turn_hi[j]));
      r->axis[j] = static_cast<uint8_t>(i);
    }
  return REFCACHE_OK;
}

int refcache_qkv_rope(const refcache_rope_t* r, const refcache_rope_rows_t* w, const void* q, int64_t ld_q, const void* k, int64_t ld_k,
                      const void* v, int64_t ld_v, void* q_out, void* k_out, void* v_out, void* stream) {
  int rc = check_rope(r, w);
  if (rc) return rc;
  rc::RopeTable t{};
  rc::RopeArgs a{};
  rope_tables(r, w, &t, &a);
  const int64_t hd = static_cast<int64_t>(w->num_heads) * r->head_dim;
  const void* src[3] = {q, k, v};
  void* dst[3] = {q_out, k_out, v_out};
  const int64_t ld[3] = {ld_q, ld_k, ld_v};
  const char* names[3] = {"q", "k", "v"};
  for (int i = 0; i < 3; ++i) {
    if ((src[i] == nullptr) != (dst[i] == nullptr)) return fail(REFCACHE_ERR_INVALID_ARG, "%s without its output, or the reverse", names[i]);
    if (!src[i]) continue;
    if ((rc = check_ld(ld[i], hd, names[i])) != 0) return rc;
    if (w->rows > 0 && ((rc = check_tensor(src[i], names[i])) != 0 || (rc = check_tensor(dst[i], "output")) != 0)) return rc;
    a.src[i] = static_cast<const uint16_t*>(src[i]);
    a.dst[i] = static_cast<uint16_t*>(dst[i]);
    a.ld[i] = ld[i];
    a.ld_dst[i] = hd;
  }
  int sms = 0;
  if ((rc = device_sms(&sms)) != 0) return rc;
  if (w->rows == 0 || (!q && !k && !v)) return REFCACHE_OK;
  const int slices = rope_slices(r, w, sms, 4, &a.head_step);
  const dim3 grid(static_cast<unsigned>(ceil_div(w->rows, rc::kRopeTokens)), static_cast<unsigned>(slices), 1);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  auto go = [&](auto kernel) { return launch_dependent(kernel, grid, dim3(rc::kRopeThreads), 0, s, t, a); };
  const cudaError_t e = r->head_dim == 128 ? (r->interleaved ? go(rc::qkv_rope_kernel<128, false>) : go(rc::qkv_rope_kernel<128, true>))
                                           : (r->interleaved ? go(rc::qkv_rope_kernel<64, false>) : go(rc::qkv_rope_kernel<64, true>));
  return e == cudaSuccess ? REFCACHE_OK : cuda_fail(e, "qkv_rope_kernel launch");
}

size_t refcache_qkv_rope_backward_bytes(const refcache_rope_t* r) {
  return r ? static_cast<size_t>(kRopeMaxParts) * 2 * 128 * sizeof(float) : 0;
}

int refcache_qkv_rope_backward(const refcache_rope_t* r, const refcache_rope_rows_t* w, const void* q, int64_t ld_q, const void* k,
                               int64_t ld_k, const void* dq_out, const void* dk_out, const void* dv_out, void* dq, int64_t ld_dq,
                               void* dk, int64_t ld_dk, void* dv, int64_t ld_dv, float* dweight_q, float* dweight_k, void* work,
                               void* stream) {
  int rc = check_rope(r, w);
  if (rc) return rc;
  rc::RopeTable t{};
  rc::RopeArgs a{};
  rope_tables(r, w, &t, &a);
  const int64_t hd = static_cast<int64_t>(w->num_heads) * r->head_dim;
  const void* src[3] = {q, k, nullptr};
  const void* grad[3] = {dq_out, dk_out, dv_out};
  void* dst[3] = {dq, dk, dv};
  float* dw[2] = {dweight_q, dweight_k};
  const int64_t ld[3] = {ld_q, ld_k, hd}, ld_dst[3] = {ld_dq, ld_dk, ld_dv};
  const char* names[3] = {"q", "k", "v"};
  for (int i = 0; i < 3; ++i) {
    if ((grad[i] == nullptr) != (dst[i] == nullptr))
      return fail(REFCACHE_ERR_INVALID_ARG, "the gradient of %s without that of its output, or the reverse", names[i]);
    const bool weighted = i < 2 && a.weight[i];
    if (i < 2 && dw[i] && !(weighted && grad[i]))
      return fail(REFCACHE_ERR_INVALID_ARG, "dweight_%s without weight_%s and the gradient of %s_out", names[i], names[i], names[i]);
    if (!grad[i]) {
      if (i < 2) a.weight[i] = nullptr;
      continue;
    }
    if ((rc = check_ld(ld_dst[i], hd, names[i])) != 0 || (weighted && (rc = check_ld(ld[i], hd, names[i])) != 0)) return rc;
    if (w->rows > 0 && ((rc = check_tensor(grad[i], names[i])) != 0 || (rc = check_tensor(dst[i], names[i])) != 0 ||
                        (weighted && (rc = check_tensor(src[i], names[i])) != 0)))
      return rc;
    a.src[i] = static_cast<const uint16_t*>(src[i]);
    a.grad[i] = static_cast<const uint16_t*>(grad[i]);
    a.dst[i] = static_cast<uint16_t*>(dst[i]);
    a.ld[i] = ld[i];
    a.ld_dst[i] = ld_dst[i];
  }
  const bool weights = a.weight[0] || a.weight[1];
  if ((rc = check_floats({dweight_q, dweight_k}, "qkv_rope_backward")) != 0) return rc;
  if (weights && (rc = check_tensor(work, "work")) != 0) return rc;
  a.dw_part = static_cast<float*>(work);
  int sms = 0;
  if ((rc = device_sms(&sms)) != 0) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  int parts = 0;
  if (w->rows > 0 && (dq_out || dk_out || dv_out)) {
    int slices = 1;
    const int blocks = rope_backward_blocks(r, w, std::min(2 * sms, kRopeMaxParts), 4, &slices, &a.head_step);
    parts = blocks * slices;
    const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(slices), 1);
    auto go = [&](auto kernel) { return launch_dependent(kernel, grid, dim3(rc::kRopeThreads), 0, s, t, a); };
    e = r->head_dim == 128
            ? (r->interleaved ? go(rc::qkv_rope_backward_kernel<128, false>) : go(rc::qkv_rope_backward_kernel<128, true>))
            : (r->interleaved ? go(rc::qkv_rope_backward_kernel<64, false>) : go(rc::qkv_rope_backward_kernel<64, true>));
    if (e != cudaSuccess) return cuda_fail(e, "qkv_rope_backward_kernel launch");
  }
  if (dweight_q || dweight_k) {
    e = launch_dependent(rc::rope_weight_grad_kernel, dim3(static_cast<unsigned>(r->head_dim / rc::kRopeSumCols), 2), dim3(1024), 0, s, static_cast<const float*>(work), parts, r->head_dim,
                         dweight_q, dweight_k);
    if (e != cudaSuccess) return cuda_fail(e, "rope_weight_grad_kernel launch");
  }
  return REFCACHE_OK;
}

int refcache_gated_norm(const refcache_gated_norm_t* p, const void* x, const void* branch, void* x_out, void* y, void* stream) {
  int rc = check_norm(p);
  if (rc) return rc;
  const int64_t rows = p->cu_rows[p->batch];
  if (rows > 0 && ((rc = check_tensor(x, "x")) != 0 || (rc = check_optional(branch, "branch")) != 0 ||
                   (rc = check_optional(x_out, "x_out")) != 0 || (rc = check_optional(y, "y")) != 0))
    return rc;
  if (rows > 0 && x_out && !branch) return fail(REFCACHE_ERR_INVALID_ARG, "x_out without a branch");
  int sms = 0;
  if ((rc = device_sms(&sms)) != 0) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const NormShape shape = norm_shape(p->width, false);
  for (int b = 0; b < p->batch; b += rc::kNormMaxSegs) {
    const int n = std::min(rc::kNormMaxSegs, p->batch - b);
    const rc::NormSegs segs = norm_segs(p, b, n);
    if (segs.cu[n] == 0) continue;
    rc::NormArgs a = norm_args(p, b, segs.cu[n]);
    const int64_t off = static_cast<int64_t>(p->cu_rows[b]) * p->width;
    a.x = static_cast<const uint16_t*>(x) + off;
    a.branch = branch ? static_cast<const uint16_t*>(branch) + off : nullptr;
    a.x_out = x_out ? static_cast<uint16_t*>(x_out) + off : nullptr;
    a.y = y ? static_cast<uint16_t*>(y) + off : nullptr;
    a.rows_per_block = norm_rows_per_block(a.rows, sms, shape);
    const int blocks = ceil_div(a.rows, a.rows_per_block);
    const cudaError_t e = with_norm_shape(shape, [&](auto nv, auto threads) {
      return launch_norm(rc::gated_norm_kernel<decltype(nv)::value, decltype(threads)::value>, shape, blocks, s, segs, a);
    });
    if (e != cudaSuccess) return cuda_fail(e, "gated_norm_kernel launch");
  }
  return REFCACHE_OK;
}

size_t refcache_gated_norm_backward_bytes(const refcache_gated_norm_t* p) {
  if (check_norm(p) != 0) return 0;
  // a slot for each block and one more for each request a block goes on to
  return static_cast<size_t>(kNormMaxBlocks + std::min(p->batch, rc::kNormMaxSegs)) * 3 * p->width * sizeof(float);
}

int refcache_gated_norm_backward(const refcache_gated_norm_t* p, const void* x_out, const void* branch, const void* dy, const void* dx_out,
                                 void* dx, void* d_branch, float* d_gate, float* d_scale, float* d_shift, float* d_weight,
                                 float* d_post_weight, void* work, void* stream) {
  int rc = check_norm(p);
  if (rc) return rc;
  const int64_t rows = p->cu_rows[p->batch];
  if (rows > 0 && ((dy && (rc = check_tensor(x_out, "x_out")) != 0) || (rc = check_optional(branch, "branch")) != 0 ||
                   (rc = check_optional(dy, "dy")) != 0 || (rc = check_optional(dx_out, "dx_out")) != 0 ||
                   (rc = check_optional(dx, "dx")) != 0 || (rc = check_optional(d_branch, "d_branch")) != 0 ||
                   (rc = check_tensor(work, "work")) != 0))
    return rc;
  // (a tensor without rows may well be NULL)
  if (rows > 0 && !branch && (d_branch || d_gate || d_post_weight))
    return fail(REFCACHE_ERR_INVALID_ARG, "gradients of the branch, its gate or its norm without a branch");
  if (rows > 0 && !dy && !dx_out) return fail(REFCACHE_ERR_INVALID_ARG, "neither dy nor dx_out");
  if ((d_weight && !p->weight) || (d_post_weight && !p->post_weight))
    return fail(REFCACHE_ERR_INVALID_ARG, "the gradient of a weight that is not there");
  if ((rc = check_floats({d_gate, d_scale, d_shift, d_weight, d_post_weight}, "gated_norm_backward")) != 0) return rc;
  int sms = 0;
  if ((rc = device_sms(&sms)) != 0) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const NormShape shape = norm_shape(p->width, true);
  for (int b = 0; b < p->batch; b += rc::kNormMaxSegs) {
    const int n = std::min(rc::kNormMaxSegs, p->batch - b);
    const rc::NormSegs segs = norm_segs(p, b, n);
    rc::NormArgs a = norm_args(p, b, segs.cu[n]);
    const int64_t off = static_cast<int64_t>(p->cu_rows[b]) * p->width;
    auto in = [&](const void* t) { return t ? static_cast<const uint16_t*>(t) + off : nullptr; };
    auto out = [&](void* t) { return t ? static_cast<uint16_t*>(t) + off : nullptr; };
    a.x = in(x_out);
    a.branch = in(branch);
    a.dy = in(dy);
    a.dx_out = in(dx_out);
    a.dx = out(dx);
    a.d_branch = out(d_branch);
    a.part = static_cast<float*>(work);
    a.rows_per_block = 1;
    cudaError_t e = cudaSuccess;
    if (a.rows > 0) {
      a.rows_per_block = ceil_div(a.rows, std::min(kNormMaxBlocks, norm_blocks(a.rows, sms, shape)));
      const int blocks = ceil_div(a.rows, a.rows_per_block);
      e = with_norm_shape(shape, [&](auto nv, auto threads) {
        return launch_norm(rc::gated_norm_backward_kernel<decltype(nv)::value, decltype(threads)::value>, shape, blocks, s, segs, a);
      });
      if (e != cudaSuccess) return cuda_fail(e, "gated_norm_backward_kernel launch");
    }
    if (!d_gate && !d_scale && !d_shift && !d_weight && !d_post_weight) continue;
    rc::NormSumArgs g{};
    auto of = [&](float* t) { return t ? t + static_cast<int64_t>(b) * p->width : nullptr; };
    g.part = a.part;
    g.d_gate = of(d_gate);
    g.d_scale = of(d_scale);
    g.d_shift = of(d_shift);
    g.d_weight = d_weight;
    g.d_post_weight = d_post_weight;
    g.gate = a.gate;
    g.scale = a.scale;
    g.weight = a.weight;
    g.post_weight = a.post_weight;
    g.ld_gate = a.ld_gate;
    g.ld_scale = a.ld_scale;
    g.width = a.width;
    g.rows_per_block = a.rows_per_block;
    g.mod_f32 = a.mod_f32;
    g.add = b > 0;
    // (by slots a request.  Call with the many and the few form: 5888 rows of 4096 in 8 requests, 37 slots each, 71 and 67
    // us, 300 of 256, 37 each, 4.7 and 11; 4608 of 8192 in 8, 19 each, 117 and 98; 5888 of 4096 in 64, 5 each, 153 and 66)
    const bool few = ceil_div(a.rows, a.rows_per_block) < 32 * n, weights = d_weight || d_post_weight;
    const dim3 grid(static_cast<unsigned>(ceil_div(p->width, few ? rc::kSumFewCols : rc::kSumCols)), 3,
                    weights ? 1u : static_cast<unsigned>(few ? ceil_div(n, rc::kSumWarps) : n));
    e = launch_dependent(few ? rc::norm_param_grad_few_kernel : rc::norm_param_grad_kernel, grid, dim3(rc::kSumThreads), 0, s, segs, g);
    if (e != cudaSuccess) return cuda_fail(e, "norm_param_grad_kernel launch");
  }
  return REFCACHE_OK;
}

size_t refcache_clip_gradients_bytes(int n) {
  if (n < 0) return 0;
  // the blocks' sums of every table, and a counter each
  return static_cast<size_t>(std::max(1, ceil_div(n, rc::kClipMaxTensors))) * (kClipMaxBlocks * sizeof(double) + 16);
}

int refcache_clip_gradients(int n, const void* const* grads, void* const* out, const int64_t* counts, const int32_t* types,
                            float max_norm, float* norm, void* work, void* stream) {
  if (n < 0 || (n > 0 && (!grads || !counts || !types))) return fail(REFCACHE_ERR_INVALID_ARG, "clip_gradients: NULL list or n < 0");
  if (!(max_norm >= 0.f)) return fail(REFCACHE_ERR_INVALID_ARG, "max_norm must be >= 0");  // (+inf: the norm alone)
  int rc = check_tensor(work, "work");
  if (rc || (rc = check_floats({norm}, "clip_gradients")) != 0) return rc;
  for (int i = 0; i < n; ++i) {
    if (counts[i] < 0) return fail(REFCACHE_ERR_INVALID_ARG, "counts[%d] is negative", i);
    if (types[i] & ~3) return fail(REFCACHE_ERR_INVALID_ARG, "types[%d] = %d is none of REFCACHE_CLIP_*", i, types[i]);
    if (counts[i] == 0) continue;
    const void* o = out ? out[i] : grads[i];
    if (!grads[i] || !o) return fail(REFCACHE_ERR_INVALID_ARG, "tensor %d is NULL", i);
    const uintptr_t gs = types[i] & 1 ? 4 : 2, os = types[i] & 2 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(grads[i]) % gs || reinterpret_cast<uintptr_t>(o) % os)
      return fail(REFCACHE_ERR_INVALID_ARG, "tensor %d is not aligned to its elements", i);
    if (!out && gs != os) return fail(REFCACHE_ERR_INVALID_ARG, "types[%d]: a tensor in place keeps its type", i);
  }
  // (of every launch, before the first)
  auto pieces_of = [](int64_t count) { return count / rc::kClipPiece + (count % rc::kClipPiece != 0); };
  for (int b = 0; b < n; b += rc::kClipMaxTensors) {
    int64_t pieces = 0;  // (512 times 2^63 / 2^14 at most)
    for (int i = b; i < std::min(n, b + rc::kClipMaxTensors); ++i) pieces += pieces_of(counts[i]);
    if (pieces >= (1ll << 31) - 1) return fail(REFCACHE_ERR_INVALID_ARG, "clip_gradients: too many elements");
  }
  int sms = 0;
  if ((rc = device_sms(&sms)) != 0) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  auto table = [&](int first) {
    rc::ClipTable t{};
    int64_t pieces = 0;
    for (int i = first; i < std::min(n, first + rc::kClipMaxTensors); ++i) {
      if (counts[i] == 0) continue;
      const int k = t.n++;
      t.g[k] = grads[i];
      t.out[k] = out ? out[i] : const_cast<void*>(grads[i]);
      t.count[k] = counts[i];
      t.types[k] = static_cast<uint8_t>(types[i]);
      t.piece0[k] = static_cast<int32_t>(pieces);
      pieces += pieces_of(counts[i]);
    }
    t.piece0[t.n] = static_cast<int32_t>(pieces);
    return t;
  };
  double* part = static_cast<double*>(work);
  int* taken = reinterpret_cast<int*>(part + static_cast<int64_t>(std::max(1, ceil_div(n, rc::kClipMaxTensors))) * kClipMaxBlocks);
  int parts = 0;
  const int resident = std::min(4 * sms, kClipMaxBlocks);
  for (int b = 0; b < n; b += rc::kClipMaxTensors) {
    const rc::ClipTable t = table(b);
    const int pieces = t.piece0[t.n];
    if (pieces == 0) continue;
    // (Pieces are dealt out in a fixed order, for the sums' sake; up to four rounds of blocks
    // even out the SMs' speeds: 906 M elements 811 us with one, 794 with four.)
    const int rounds = std::max(1, std::min(pieces / (8 * resident), kClipMaxBlocks / resident));
    const int grid = std::min(pieces, std::min(4, rounds) * resident);
    const cudaError_t e =
        launch_dependent(rc::clip_norm_kernel, dim3(static_cast<unsigned>(grid)), dim3(rc::kClipThreads), 0, s, t, part + parts, taken + 4 * (b / rc::kClipMaxTensors));
    if (e != cudaSuccess) return cuda_fail(e, "clip_norm_kernel launch");
    parts += grid;
  }
  const bool scale = !std::isinf(max_norm) || out != nullptr;  // an infinite bound in place leaves the tensors as they are
  for (int b = 0; b == 0 || (b < n && scale); b += rc::kClipMaxTensors) {
    rc::ClipTable t = table(b);
    if (!scale) t.n = 0, t.piece0[0] = 0;
    const int grid = std::max(1, std::min(t.piece0[t.n], resident));
    const cudaError_t e = launch_dependent(rc::clip_scale_kernel, dim3(static_cast<unsigned>(grid)), dim3(rc::kClipThreads), 0, s, t,
                                           static_cast<const double*>(part), parts, taken + 4 * (b / rc::kClipMaxTensors), max_norm, b == 0 ? norm : nullptr, out == nullptr ? 1 : 0);
    if (e != cudaSuccess) return cuda_fail(e, "clip_scale_kernel launch");
  }
  return REFCACHE_OK;
}

}  // extern "C"
