// f8_ops.cu -- the entry points of include/refcache.h for linear layers in 8 bits:
// rows and weights into their 8-bit form (f8_rows.cuh), products on it (f8_linear.cuh, f8_few.cuh, f8_wgrad.cuh).
// Argument checks and launches; no call allocates memory.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "refcache.h"
#include "f8_few.cuh"
#include "f8_linear.cuh"
#include "f8_rows.cuh"
#include "f8_wgrad.cuh"
#include "host_common.h"

using rc_host::aligned16;
using rc_host::cuda_fail;
using rc_host::device_sms;
using rc_host::fail;
using rc_host::launch_dependent;

namespace {

constexpr int64_t kMaxRows = (1ll << 31) - 1 - 512;
constexpr int kMaxWidth = 1 << 20;

unsigned ceil_div(int64_t a, int64_t b) { return static_cast<unsigned>((a + b - 1) / b); }

int check_tensor(const void* p, const char* name) {
  if (!p) return fail(REFCACHE_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned16(p)) return fail(REFCACHE_ERR_INVALID_ARG, "%s: tensor pointer not 16-byte aligned", name);
  return REFCACHE_OK;
}
int check_width(int64_t width, const char* name) {
  if (width < 16 || width > kMaxWidth || width % 16)
    return fail(REFCACHE_ERR_INVALID_ARG, "%s: widths are multiples of 16 from 16 to %d (got %lld)", name, kMaxWidth, static_cast<long long>(width));
  return REFCACHE_OK;
}
int check_ld(int64_t ld, int64_t width, const char* name) {
  if (ld < width || ld % 8 || ld > (1ll << 32))
    return fail(REFCACHE_ERR_INVALID_ARG, "%s: %lld elements between rows of %lld (a multiple of 8, at least the width)", name,
                static_cast<long long>(ld), static_cast<long long>(width));
  return REFCACHE_OK;
}
// Rows in 8-bit form (of `width`, unless it is 0).
int check_rows(const refcache_f8_rows_t* r, int64_t rows, int width, const char* name) {
  if (!r) return fail(REFCACHE_ERR_INVALID_ARG, "%s is NULL", name);
  int rc = check_width(r->width, name);
  if (rc) return rc;
  if (r->rows < 0 || r->rows > kMaxRows) return fail(REFCACHE_ERR_INVALID_ARG, "%s: %lld rows", name, static_cast<long long>(r->rows));
  if (width && r->width != width) return fail(REFCACHE_ERR_INVALID_ARG, "%s: width %d, expected %d", name, r->width, width);
  if (rows >= 0 && r->rows != rows)
    return fail(REFCACHE_ERR_INVALID_ARG, "%s: %lld rows, expected %lld", name, static_cast<long long>(r->rows), static_cast<long long>(rows));
  if (r->rows > 0 && ((rc = check_tensor(r->codes, name)) != 0 || (rc = check_tensor(r->scales, name)) != 0 ||
                      (rc = check_tensor(r->tiles, name)) != 0))
    return rc;
  return REFCACHE_OK;
}
int check_weight(const refcache_f8_weight_t* w, bool plain, bool transposed) {
  if (!w) return fail(REFCACHE_ERR_INVALID_ARG, "weight is NULL");
  int rc;
  if ((rc = check_width(w->out_width, "weight")) != 0 || (rc = check_width(w->in_width, "weight")) != 0) return rc;
  if (plain && ((rc = check_tensor(w->codes, "weight codes")) != 0 || (rc = check_tensor(w->scales, "weight scales")) != 0 ||
                (rc = check_tensor(w->tiles, "weight tiles")) != 0))
    return rc;
  if (transposed && ((rc = check_tensor(w->codes_t, "weight codes_t")) != 0 || (rc = check_tensor(w->scales_t, "weight scales_t")) != 0 ||
                     (rc = check_tensor(w->tiles_t, "weight tiles_t")) != 0))
    return rc;
  return REFCACHE_OK;
}
int check_bias(const void* bias, int f32) {
  if (bias && (reinterpret_cast<uintptr_t>(bias) & (f32 ? 3u : 1u))) return fail(REFCACHE_ERR_INVALID_ARG, "bias is not aligned");
  return REFCACHE_OK;
}

rc::f8::Rows rows_of(void* codes, void* scales, void* tiles, int64_t rows, int width) {
  return {static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales), static_cast<uint8_t*>(tiles), rows, width, REFCACHE_F8_PITCH(width),
          static_cast<int32_t>(ceil_div(rows, 128))};
}
rc::f8::Rows rows_of(const refcache_f8_rows_t* r) { return r ? rows_of(r->codes, r->scales, r->tiles, r->rows, r->width) : rc::f8::Rows{}; }
rc::f8::Rows rows_of(const refcache_f8_weight_t* w, bool transposed) {
  return transposed ? rows_of(w->codes_t, w->scales_t, w->tiles_t, w->in_width, w->out_width)
                    : rows_of(w->codes, w->scales, w->tiles, w->out_width, w->in_width);
}

// Memory that a call reads or writes: outputs lie apart from inputs and from each other.
struct Spans {
  struct {
    uintptr_t first, last;
  } of[9];
  int n = 0;
  Spans& add(const void* p, int64_t bytes) {
    if (p && bytes > 0) of[n++] = {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes};
    return *this;
  }
  Spans& add(const rc::f8::Rows& r) { return add(r.codes, r.rows * r.width).add(r.scales, r.rows * r.pitch).add(r.tiles, r.pitch / 4 * 512ll * r.chunks); }
  Spans& add(const refcache_f8_rows_t* r) { return add(rows_of(r)); }
  // (a weight has a row of scales for each 128)
  Spans& add(const refcache_f8_weight_t* w, bool transposed) {
    rc::f8::Rows r = rows_of(w, transposed);
    add(r.codes, r.rows * r.width).add(r.tiles, r.pitch / 4 * 512ll * r.chunks);
    return add(r.scales, static_cast<int64_t>(r.chunks) * r.pitch);
  }
  // Of rows that lie apart the first one alone: between them there may be anything.
  Spans& add_bf16(const void* p, int64_t rows, int64_t width, int64_t ld) { return add(p, rows > 0 ? 2 * width * (ld == width ? rows : 1) : 0); }
};
int check_apart(const Spans& out, const Spans& in) {
  for (int i = 0; i < out.n; ++i) {
    auto meets = [&](const Spans& o, int n) {
      for (int j = 0; j < n; ++j)
        if (out.of[i].first < o.of[j].last && o.of[j].first < out.of[i].last) return true;
      return false;
    };
    if (meets(out, i) || meets(in, in.n)) return fail(REFCACHE_ERR_INVALID_ARG, "an output overlaps an input or another output");
  }
  return REFCACHE_OK;
}

// CTA pairs of a kernel that run at once on the current device; sets its attributes on first use.
template <typename Kernel>
int pairs_of(Kernel kernel, std::atomic<int>& kept, int threads, uint32_t smem, int sms, int* pairs) {
  int n = kept.load();
  if (n == 0) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(f8)");
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2 * static_cast<unsigned>(sms / 2));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
    if (e != cudaSuccess) return cuda_fail(e, "cudaOccupancyMaxActiveClusters(f8)");
    if (n < 1) return fail(REFCACHE_ERR_CUDA, "no CTA pair of an 8-bit product fits on the device");
    kept.store(n);
  }
  *pairs = n;
  return REFCACHE_OK;
}

// How a product is taken apart: tiles of 256 rows over CTA pairs, `bn` columns each, or (few) the
// weight streamed by clusters of `splits` CTAs.  Of tiles of 256 columns, those behind the last full round over
// the pairs may be taken in pieces of `tail` columns (64 or 128), if that makes no second round.
struct LinearPlan {
  bool few;
  int bn, tail;
  int64_t whole, items;  // tiles that are not in pieces; these and the pieces
  int splits, per;
};

// By estimated cycles, whose constants are fitted to calls one behind the other (microseconds, on weights from memory):
//   rows x out x in       pairs   few, splits 1 / 2 / 3 / 4 / 8
//   2 x 24576 x 4096      35.9    21.0 / 25.4 / 23.7 / 26.2 / 38.8
//   2 x 4096 x 4096       14.4    16.3 /  9.9 /  8.4 /  7.0 /  6.4
//   64 x 4096 x 16384     37.7    60.1 / 33.6 / 25.7 / 21.1 / 18.1
//   200 x 2048 x 8192     20.7    35.8 / 22.3 / 19.1 / 16.0 / 14.9
//   300 x 4096 x 4096     13.2    22.2 / 18.7 / 16.6 / 22.3 / 31.0
// Pairs: rounds of tiles; a block of 128 columns of x takes a pair 2 bn cycles of MMAs, or (256 + bn) for its
// loads, 16 KB + 64 bn bytes to each CTA (a fit: in long rows a stage takes more of both, f8_linear.cuh); a weight of which
// every tile is read once comes at 1800 bytes a cycle.  Few: the weight at 3300 bytes a cycle, all that the CTAs load at
// 5500, and a CTA's own loads at 24.
LinearPlan plan_linear(int64_t rows, int width, int k, int pairs, int sms, int step) {
  const int64_t blocks = ceil_div(k, 128);
  LinearPlan best{};
  int64_t least = -1;
  for (int bn = step; bn <= 256; bn += step) {
    const int64_t tiles = static_cast<int64_t>(ceil_div(rows, 256)) * ceil_div(width, bn), over = tiles % pairs;
    for (int tail = bn == 256 && tiles > pairs ? step : bn; tail <= bn; tail *= 2) {
      if (tail < bn && (over == 0 || over * (bn / tail) > pairs)) continue;
      const int64_t rounds = tiles / pairs * (blocks * (256 + bn) + 700) + (over ? blocks * (256 + tail) + 700 : 0);
      const int64_t cost = 8000 + std::max(rounds, static_cast<int64_t>(width) * k / 1800);
      if (least < 0 || cost < least || (cost == least && tail == bn))
        least = cost, best = {false, bn, tail, tail < bn ? tiles - over : tiles, tail < bn ? tiles - over + over * (bn / tail) : tiles, 1, 0};
    }
  }
  if (rows > 128 * 65535ll || ceil_div(width, 128) > 65535) return best;
  const int64_t wide = ceil_div(width, 128), tiles = wide * ceil_div(rows, 128);
  const int64_t bytes = rc::f8::FewSmem::slot_bytes(rc::f8::FewSmem::rows_of_tile(rows));
  for (int s = 1; s <= 8; ++s) {
    const int64_t per = (blocks + 4 * s - 1) / (4 * s) * 4;
    if ((blocks + per - 1) / per != s) continue;
    const int64_t waves = (tiles * s + 2 * sms - 1) / (2 * sms);
    const int64_t cost = 6000 + 1700 * waves + std::max({wide * blocks * rc::f8::FewSmem::kA / 3300, tiles * blocks * bytes / 5500, waves * per * bytes / 24});
    if (cost <= least) least = cost, best = {true, 128, 128, 0, 0, s, static_cast<int>(per)};
  }
  return best;
}

int tiles_map(CUtensorMap* m, const rc::f8::Rows& r) {
  return rc_host::encode_lines(m, r.tiles, static_cast<int64_t>(r.pitch / 4) * r.chunks);
}

template <int kEpi, bool kLong>
int launch_few(const LinearPlan& p, const rc::f8::Rows& x, const rc::f8::Rows& w, const rc::f8::Out& o, int* status, int dev, void* stream) {
  using L = rc::f8::FewSmem;
  static std::atomic<bool> set[rc_host::kMaxDevices];
  if (!set[dev].load()) {
    const cudaError_t e = cudaFuncSetAttribute(rc::f8::f8_few_kernel<kEpi, kLong>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kDynamic);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(f8_few_kernel)");
    set[dev].store(true);
  }
  rc::f8::FewArgs a{};
  a.o = o;
  a.x_chunks = x.chunks, a.w_chunks = w.chunks;
  a.k = x.width, a.per = p.per;
  const int n = L::rows_of_tile(o.rows);
  a.n = n, a.slots = std::min<int>(L::kMaxSlots, L::kStages / L::slot_bytes(n));
  a.guard.status = status;
  a.guard.timeout_ns = rc_host::wait_timeout_ns();
  rc::f8::LinearMaps maps;
  int rc;
  if ((rc = rc_host::encode_map(&maps.x, x.codes, x.width, x.rows, x.width, static_cast<uint32_t>(n))) != 0 ||
      (rc = rc_host::encode_map(&maps.w, w.codes, w.width, w.rows, w.width, 128)) != 0 ||
      (rc = tiles_map(&maps.x_tiles, x)) != 0 || (rc = tiles_map(&maps.w_tiles, w)) != 0)
    return rc;
  a.guard.stop = rc_host::take_debug_stop();
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(p.splits), ceil_div(o.width, 128), ceil_div(o.rows, 128));
  cfg.blockDim = dim3(L::kThreads);
  cfg.dynamicSmemBytes = L::kDynamic;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(p.splits);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cudaError_t e = cudaLaunchKernelEx(&cfg, rc::f8::f8_few_kernel<kEpi, kLong>, maps, a);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? REFCACHE_OK : cuda_fail(e, "f8_few_kernel launch");
}

template <int kEpi, bool kLong>
int launch_linear_of(const rc::f8::Rows& x, const rc::f8::Rows& w, const rc::f8::Out& o, void* stream) {
  using L = rc::f8::LinearSmem;
  if (o.rows == 0) return REFCACHE_OK;
  static std::atomic<int> kept[rc_host::kMaxDevices];
  int sms = 0, dev = 0, pairs = 0;
  rc::f8::LinearArgs a{};
  int rc = device_sms(&sms);
  if (rc || (rc = rc_host::device_status_word(&dev, &a.guard.status)) != 0 ||
      (rc = pairs_of(rc::f8::f8_linear_kernel<kEpi, kLong>, kept[dev], L::kThreads, L::kDynamic, sms, &pairs)) != 0)
    return rc;
  const LinearPlan p = plan_linear(o.rows, o.width, x.width, pairs, sms, kEpi < rc::f8::kGelu ? 64 : 128);
  constexpr int kFew = kEpi == rc::f8::kStoreLines ? rc::f8::kStore : kEpi;
  if (p.few && kLong && p.per > rc::f8::kSumBlocks) return launch_few<kFew, kLong>(p, x, w, o, a.guard.status, dev, stream);
  if (p.few) return launch_few<kFew, false>(p, x, w, o, a.guard.status, dev, stream);
  a.o = o;
  a.x_chunks = x.chunks, a.w_chunks = w.chunks;
  a.k = x.width;
  a.bn = p.bn;
  const int64_t tiles_m = ceil_div(o.rows, 256), tiles_n = ceil_div(o.width, a.bn);
  a.tail = p.tail;
  if (tiles_m * tiles_n > (1ll << 30)) return fail(REFCACHE_ERR_INVALID_ARG, "too many rows for a width of %d", o.width);
  a.tiles = {static_cast<int32_t>(tiles_m), static_cast<int32_t>(tiles_n)};
  a.n_whole = static_cast<int32_t>(p.whole), a.n_items = static_cast<int32_t>(p.items);
  a.guard.timeout_ns = rc_host::wait_timeout_ns();
  rc::f8::LinearMaps maps;
  if ((rc = rc_host::encode_map(&maps.x, x.codes, x.width, x.rows, x.width, 128)) != 0 ||
      (rc = rc_host::encode_map(&maps.w, w.codes, w.width, w.rows, w.width, static_cast<uint32_t>(a.bn / 2))) != 0 ||
      (rc = rc_host::encode_map(&maps.w_tail, w.codes, w.width, w.rows, w.width, static_cast<uint32_t>(a.tail / 2))) != 0 ||
      (rc = tiles_map(&maps.x_tiles, x)) != 0 || (rc = tiles_map(&maps.w_tiles, w)) != 0)
    return rc;
  a.guard.stop = rc_host::take_debug_stop();
  const unsigned clusters = static_cast<unsigned>(std::min<int64_t>(p.items, pairs));
  const cudaError_t e = launch_dependent(rc::f8::f8_linear_kernel<kEpi, kLong>, dim3(2 * clusters), dim3(L::kThreads), L::kDynamic,
                                         static_cast<cudaStream_t>(stream), maps, a);
  return e == cudaSuccess ? REFCACHE_OK : cuda_fail(e, "f8_linear_kernel launch");
}

template <int kEpi>
int launch_linear(const rc::f8::Rows& x, const rc::f8::Rows& w, const rc::f8::Out& o, void* stream) {
  static_assert(kEpi != rc::f8::kStoreLines || rc::f8::kLinesMost <= rc::f8::kBlock * rc::f8::kSumBlocks, "lines of long rows");
  if (kEpi != rc::f8::kStoreLines && x.width > rc::f8::kBlock * rc::f8::kSumBlocks)
    return launch_linear_of<kEpi == rc::f8::kStoreLines ? rc::f8::kStore : kEpi, true>(x, w, o, stream);
  return launch_linear_of<kEpi, false>(x, w, o, stream);
}

// How a weight gradient is taken apart.
struct WgradPlan {
  int panel;  // columns of x whose values are in the workspace at a time
  int bn, stages, splits, per_split;
  size_t values_bytes, parts_bytes;
};
constexpr int64_t kPanelBytes = 256ll << 20;  // of a panel, unless 256 columns are more

// The plan is for the 76 CTA pairs of a GB300, whatever the device has to spare, so that a workspace's size
// does not depend on it.  Cycles by rounds of items over the pairs: a stage of 64 rows takes 2 bn of
// MMAs or 256 + bn to move its operands, a tile about 1000 at its ends; parts have to be written and
// read again, at about 3.5 KB a cycle, by another kernel (5000).
WgradPlan plan_wgrad(int64_t rows, int n, int k) {
  constexpr int kPairs = 76;
  WgradPlan best{};
  const int64_t fit = std::max<int64_t>(kPanelBytes / (2 * std::max<int64_t>(rows, 1)) / 256 * 256, 256);
  const int panel = static_cast<int>(std::min<int64_t>(fit, k));
  int64_t least = -1;
  for (int bn = n > 128 ? 256 : 128; bn >= 128; bn -= 128) {
    WgradPlan p{};
    p.panel = panel, p.bn = bn;
    p.stages = static_cast<int>((rows + 63) / 64);
    const int64_t tiles = static_cast<int64_t>(ceil_div(n, bn)) * ceil_div(panel, 256);
    for (int s = 1; s <= 32; ++s) {
      if (s > 1 && (panel < k || s > p.stages || s * tiles > kPairs)) break;
      p.per_split = static_cast<int>(ceil_div(p.stages, s));
      p.splits = p.per_split ? static_cast<int>(ceil_div(p.stages, p.per_split)) : 1;
      const int64_t rounds = (p.splits * tiles + kPairs - 1) / kPairs;
      const int64_t cost = rounds * (static_cast<int64_t>(p.per_split) * std::max(2 * bn, 256 + bn) + 1000) +
                           (p.splits > 1 ? 5000 + (p.splits + 1ll) * n * k * 4 / 3500 : 0);
      if (least < 0 || cost < least) least = cost, best = p;
    }
  }
  best.values_bytes = (static_cast<size_t>(rows) * panel * 2 + 255) / 256 * 256;
  best.parts_bytes = best.splits > 1 ? static_cast<size_t>(best.splits) * n * k * sizeof(float) : 0;
  return best;
}

}  // namespace

extern "C" {

int refcache_f8_quantize(const void* x, int64_t ld, const refcache_f8_rows_t* out, void* stream) {
  int rc = check_rows(out, -1, 0, "out");
  if (rc || (rc = check_ld(ld, out->width, "x")) != 0) return rc;
  if (out->rows == 0) return REFCACHE_OK;
  if ((rc = check_tensor(x, "x")) != 0 || (rc = check_apart(Spans().add(out), Spans().add_bf16(x, out->rows, out->width, ld))) != 0) return rc;
  int sms = 0;
  if ((rc = device_sms(&sms)) != 0) return rc;
  const int strips = out->width > 512 ? 4 : out->width > 256 ? 2 : 1;
  const int64_t warps = (out->rows + 4 / strips - 1) / (4 / strips) * ceil_div(out->width, 256 * strips);
  const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((warps + rc::f8::kRowsThreads / 32 - 1) / (rc::f8::kRowsThreads / 32), 32ll * sms));
  auto go = [&](auto kernel) {
    return launch_dependent(kernel, dim3(blocks), dim3(rc::f8::kRowsThreads), 0, static_cast<cudaStream_t>(stream), static_cast<const uint16_t*>(x), ld, rows_of(out));
  };
  const cudaError_t e = strips == 4 ? go(rc::f8::f8_quantize_kernel<4>) : strips == 2 ? go(rc::f8::f8_quantize_kernel<2>) : go(rc::f8::f8_quantize_kernel<1>);
  return e == cudaSuccess ? REFCACHE_OK : cuda_fail(e, "f8_quantize launch");
}

int refcache_f8_quantize_weight(const void* w, int w_f32, const refcache_f8_weight_t* out, void* stream) {
  const bool both = out && (out->codes_t || out->scales_t || out->tiles_t);
  int rc = check_weight(out, true, both);
  if (rc || (rc = check_tensor(w, "w")) != 0) return rc;
  Spans outs;
  outs.add(out, false);
  if (both) outs.add(out, true);
  if ((rc = check_apart(outs, Spans().add(w, static_cast<int64_t>(out->out_width) * out->in_width * (w_f32 ? 4 : 2)))) != 0) return rc;
  int sms = 0;
  if ((rc = device_sms(&sms)) != 0) return rc;
  const rc::f8::Rows t = both ? rows_of(out, true) : rc::f8::Rows{};
  const dim3 grid(ceil_div(out->in_width, 128), ceil_div(out->out_width, 128));
  auto go = [&](auto kernel) { return launch_dependent(kernel, grid, dim3(256), 0, static_cast<cudaStream_t>(stream), w, rows_of(out, false), t); };
  const cudaError_t e = w_f32 ? go(rc::f8::f8_quantize_weight_kernel<true>) : go(rc::f8::f8_quantize_weight_kernel<false>);
  return e == cudaSuccess ? REFCACHE_OK : cuda_fail(e, "f8_quantize_weight launch");
}

int refcache_f8_linear(const refcache_f8_rows_t* x, const refcache_f8_weight_t* w, int transposed, const void* bias, int bias_f32, void* y,
                       int64_t ld_y, void* stream) {
  const bool t = transposed != 0;
  int rc = check_weight(w, !t, t);
  if (rc) return rc;
  const int in = t ? w->out_width : w->in_width, out = t ? w->in_width : w->out_width;
  if ((rc = check_rows(x, -1, in, "x")) != 0 || (rc = check_bias(bias, bias_f32)) != 0 || (rc = check_ld(ld_y, out, "y")) != 0) return rc;
  if (x->rows > 0 && (rc = check_tensor(y, "y")) != 0) return rc;
  if ((rc = check_apart(Spans().add_bf16(y, x->rows, out, ld_y), Spans().add(x).add(w, t).add(bias, static_cast<int64_t>(out) * (bias_f32 ? 4 : 2)))) != 0) return rc;
  rc::f8::Out o{};
  o.bias = bias, o.bias_f32 = bias_f32, o.width = out, o.rows = x->rows;
  o.y = static_cast<uint16_t*>(y), o.ld = ld_y;
  return in <= rc::f8::kLinesMost ? launch_linear<rc::f8::kStoreLines>(rows_of(x), rows_of(w, t), o, stream)
                                  : launch_linear<rc::f8::kStore>(rows_of(x), rows_of(w, t), o, stream);
}

int refcache_f8_linear_gelu(const refcache_f8_rows_t* x, const refcache_f8_weight_t* w, const void* bias, int bias_f32, int form,
                            const refcache_f8_rows_t* a, const refcache_f8_rows_t* u8, void* stream) {
  int rc = check_weight(w, true, false);
  if (rc || (rc = check_rows(x, -1, w->in_width, "x")) != 0 || (rc = check_rows(a, x->rows, w->out_width, "a")) != 0 ||
      (u8 && (rc = check_rows(u8, x->rows, w->out_width, "u8")) != 0) || (rc = check_bias(bias, bias_f32)) != 0)
    return rc;
  if (form != REFCACHE_GELU_ERF && form != REFCACHE_GELU_TANH) return fail(REFCACHE_ERR_INVALID_ARG, "unknown form %d of the GELU", form);
  if ((rc = check_apart(Spans().add(a).add(u8), Spans().add(x).add(w, false).add(bias, static_cast<int64_t>(w->out_width) * (bias_f32 ? 4 : 2)))) != 0) return rc;
  rc::f8::Out o{};
  o.bias = bias, o.bias_f32 = bias_f32, o.width = w->out_width, o.rows = x->rows;
  o.a = rows_of(a), o.u = rows_of(u8);
  return form == REFCACHE_GELU_ERF ? launch_linear<rc::f8::kGelu>(rows_of(x), rows_of(w, false), o, stream)
                                   : launch_linear<rc::f8::kGelu + 1>(rows_of(x), rows_of(w, false), o, stream);
}

int refcache_f8_linear_gelu_backward(const refcache_f8_rows_t* dy, const refcache_f8_weight_t* w, int form, const refcache_f8_rows_t* u8,
                                     void* du, int64_t ld_du, const refcache_f8_rows_t* du8, void* stream) {
  int rc = check_weight(w, false, true);
  if (rc || (rc = check_rows(dy, -1, w->out_width, "dy")) != 0 || (rc = check_rows(u8, dy->rows, w->in_width, "u8")) != 0 ||
      (du8 && (rc = check_rows(du8, dy->rows, w->in_width, "du8")) != 0))
    return rc;
  if (form != REFCACHE_GELU_ERF && form != REFCACHE_GELU_TANH) return fail(REFCACHE_ERR_INVALID_ARG, "unknown form %d of the GELU", form);
  if (!du && !du8) return fail(REFCACHE_ERR_INVALID_ARG, "neither du nor du8 is given");
  if (du && ((rc = check_tensor(du, "du")) != 0 || (rc = check_ld(ld_du, w->in_width, "du")) != 0)) return rc;
  if ((rc = check_apart(Spans().add_bf16(du, dy->rows, w->in_width, ld_du).add(du8), Spans().add(dy).add(u8).add(w, true))) != 0) return rc;
  rc::f8::Out o{};
  o.width = w->in_width, o.rows = dy->rows;
  o.y = static_cast<uint16_t*>(du), o.ld = ld_du;
  o.a = rows_of(du8), o.u = rows_of(u8);
  return form == REFCACHE_GELU_ERF ? launch_linear<rc::f8::kGeluGrad>(rows_of(dy), rows_of(w, true), o, stream)
                                   : launch_linear<rc::f8::kGeluGrad + 1>(rows_of(dy), rows_of(w, true), o, stream);
}

size_t refcache_f8_weight_grad_bytes(int64_t rows, int out_width, int in_width) {
  if (rows <= 0 || rows > kMaxRows || check_width(out_width, "dw") != 0 || check_width(in_width, "dw") != 0) return 0;
  const WgradPlan p = plan_wgrad(rows, out_width, in_width);
  return p.values_bytes + p.parts_bytes;
}

int refcache_f8_weight_grad(const void* dy, int64_t ld_dy, const refcache_f8_rows_t* x, int out_width, const void* add, void* dw, int dw_f32,
                            float* d_bias, void* work, void* stream) {
  using L = rc::f8::WgradSmem;
  int rc = check_rows(x, -1, 0, "x");
  if (rc || (rc = check_width(out_width, "dy")) != 0 || (rc = check_ld(ld_dy, out_width, "dy")) != 0 || (rc = check_tensor(dw, "dw")) != 0 ||
      (add && (rc = check_tensor(add, "add")) != 0) || (x->rows > 0 && (rc = check_tensor(dy, "dy")) != 0))
    return rc;
  if (reinterpret_cast<uintptr_t>(d_bias) & 3u) return fail(REFCACHE_ERR_INVALID_ARG, "d_bias is not 4-byte aligned");
  const int n = out_width, k = x->width;
  const WgradPlan p = plan_wgrad(x->rows, n, k);
  if (x->rows > 0 && (rc = check_tensor(work, "work")) != 0) return rc;
  const int64_t dw_bytes = static_cast<int64_t>(n) * k * (dw_f32 ? 4 : 2);
  Spans outs, ins;
  outs.add(dw, dw_bytes).add(d_bias, 4ll * n).add(work, x->rows > 0 ? static_cast<int64_t>(p.values_bytes + p.parts_bytes) : 0);
  ins.add_bf16(dy, x->rows, n, ld_dy).add(x);
  if (add != dw) ins.add(add, dw_bytes);
  if ((rc = check_apart(outs, ins)) != 0) return rc;
  static std::atomic<int> kept[rc_host::kMaxDevices];
  rc::f8::WgradArgs a{};
  int sms = 0, dev = 0, pairs = 0;
  if ((rc = device_sms(&sms)) != 0 || (rc = rc_host::device_status_word(&dev, &a.guard.status)) != 0 ||
      (rc = pairs_of(rc::f8::f8_wgrad_kernel, kept[dev], L::kThreads, L::kDynamic, sms, &pairs)) != 0)
    return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  float* parts = reinterpret_cast<float*>(static_cast<uint8_t*>(work) + p.values_bytes);
  a.guard.stop = rc_host::take_debug_stop();
  a.guard.timeout_ns = rc_host::wait_timeout_ns();
  const rc::f8::Rows r = rows_of(x);
  auto inputs = [&](int col0, int cols) {
    constexpr int kThreads = rc::f8::kInputThreads, kBlocks = rc::f8::kInputBlocks;
    const int64_t strips = r.rows * (cols / 16);
    const unsigned bias = d_bias && col0 == 0 ? ceil_div(n, 64) : 0;
    const unsigned values = ceil_div(std::min<int64_t>(ceil_div(strips, kThreads), 16ll * sms), kBlocks);
    e = launch_dependent(rc::f8::f8_wgrad_inputs_kernel, dim3(kBlocks * (bias + values)), dim3(kThreads), 0, s, r, col0, cols,
                         static_cast<uint16_t*>(work), static_cast<const uint16_t*>(dy), ld_dy, n, d_bias, static_cast<int>(bias));
    return e == cudaSuccess ? REFCACHE_OK : cuda_fail(e, "f8_wgrad_inputs_kernel launch");
  };
  if (x->rows == 0 && d_bias && (rc = inputs(0, 0)) != 0) return rc;
  for (int col0 = 0; x->rows > 0 && col0 < k; col0 += p.panel) {
    const int cols = std::min(p.panel, k - col0);
    const int64_t size = dw_f32 ? 4 : 2;
    a.add = add ? static_cast<const uint8_t*>(add) + col0 * size : nullptr;
    a.dw = p.splits > 1 ? static_cast<void*>(parts) : static_cast<uint8_t*>(dw) + col0 * size;
    a.ld = k, a.f32 = p.splits > 1 || dw_f32;
    a.n = n, a.k = cols, a.bn = p.bn;
    a.stages = p.stages, a.splits = p.splits, a.per_split = p.per_split;
    a.tiles = {static_cast<int32_t>(ceil_div(n, p.bn)), static_cast<int32_t>(ceil_div(cols, 256))};
    const int tiles = a.tiles.m * a.tiles.n * p.splits, over = tiles % pairs;
    const bool halves = p.splits == 1 && p.bn == 256 && tiles > pairs && 2 * over <= pairs;
    a.n_whole = halves ? tiles - over : tiles, a.n_items = halves ? tiles + over : tiles;
    rc::f8::WgradMaps maps;
    if ((rc = rc_host::encode_map(&maps.dy, dy, 2 * static_cast<int64_t>(n), r.rows, 2 * ld_dy, 64)) != 0 ||
        (rc = rc_host::encode_map(&maps.x, work, 2 * static_cast<int64_t>(cols), r.rows, 2 * static_cast<int64_t>(cols), 64)) != 0)
      return rc;
    if ((rc = inputs(col0, cols)) != 0) return rc;
    const unsigned clusters = static_cast<unsigned>(std::min(a.n_items, pairs));
    e = launch_dependent(rc::f8::f8_wgrad_kernel, dim3(2 * clusters), dim3(L::kThreads), L::kDynamic, s, maps, a);
    if (e != cudaSuccess) return cuda_fail(e, "f8_wgrad_kernel launch");
  }
  if (x->rows == 0 || p.splits > 1) {
    const int64_t count = static_cast<int64_t>(n) * k;
    const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((count + 2047) / 2048, 8ll * sms));
    e = launch_dependent(rc::f8::f8_wgrad_sum_kernel, dim3(blocks), dim3(256), 0, s, static_cast<const float*>(parts), x->rows == 0 ? 0 : p.splits,
                         count, add, dw, dw_f32);
    if (e != cudaSuccess) return cuda_fail(e, "f8_wgrad_sum_kernel launch");
  }
  return REFCACHE_OK;
}

}  // extern "C"
