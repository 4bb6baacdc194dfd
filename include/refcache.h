/*
 * refcache.h -- C ABI of the beyond-mask joint attention library for GB300
 * (sm_103a): exact reference K/V caching with static text anchors.
 *
 * The paper's method (Sec. 3.3 "Static Text Anchors", App. C "Derivation"):
 * one request's in-context sequence is [LT, X_t, ST, R] -- live instruction
 * text, the denoising target, static text anchors (the instruction embedded
 * once at t = 0) and the tokens of K reference images R = [R(1); ...; R(K)]
 * (Eq. 1).  R and ST attend each other and nothing else, so their layerwise
 * K and V (Eq. 2) never depend on X_t and are computed once; the live rows
 * [LT, X_t] attend [LT, X_t, R] at every denoising step.
 *
 *   refcache_build   the one-shot static prefill: rows [ST; R] attend keys
 *                    [ST; R]; the R rows' K and V are written into the
 *                    persistent per-layer cache (Sec. 3.3, Eq. cost-pre).
 *   step_attention   one layer of one denoising step: rows [LT; X_t] attend
 *                    their own keys and the cached R keys (App. C, Eq.
 *                    cost-step); no mask is materialised.
 *   full_attention   the full-attention recompute every key of [LT; X_t; R]
 *                    visible to every row (Sec. 3.2, C_full in App. C): the
 *                    baseline the cache is measured against.
 *
 * For training the students that the paper distils (Sec. 3.4), and for the block
 * around the attention: the three calls' gradients (*_backward), the way from a
 * projection's rows to the attention's q, k and v (refcache_qkv_rope), the gated
 * residual with the norm behind it (refcache_gated_norm), both with their
 * gradients, the clipping of gradients (refcache_clip_gradients), and the linear
 * layers of the block in 8 bits, whose inputs stay as they are for the backward
 * pass (refcache_f8_*).
 *
 * Conventions shared by every entry point
 *   - Tensors are THD: [tokens, num_heads, head_dim] bf16, head_dim
 *     contiguous, rows of consecutive requests packed back to back.  Base
 *     pointers must be device pointers aligned to 16 bytes.
 *   - head_dim is 64 or 128; num_heads >= 1.
 *   - Every input row must hold finite values (rows of a neighbouring request
 *     may be read into a tile and masked out; they must not be NaN/Inf).
 *   - softmax_scale must be finite and > 0 (1/sqrt(head_dim) is the usual
 *     choice; the paper does not state it).
 *   - lse outputs are optional (NULL = not written): fp32 [tokens, num_heads],
 *     natural-log log-sum-exp of the scaled scores of each row.
 *   - Outputs are bf16 rounded to nearest-even; scores, softmax and
 *     accumulation are fp32; P is rounded to bf16 before the P.V product.
 *   - Calls are asynchronous on `stream` (a cudaStream_t passed as void*;
 *     NULL = legacy default stream) and return a status code below.  A
 *     non-zero return means nothing was launched.  Device-side faults of a
 *     launched kernel (a bounded wait that ran out) are reported later by
 *     refcache_status().
 *   - Host arrays (segment tables) are read during the call only; the library
 *     keeps its own copies.
 *   - No entry point allocates device memory except refcache_create (the
 *     cache, unless it is given memory, and a separate work
 *     list with a workspace for split items, see refcache_create) and
 *     full_attention (a per-device work-list buffer that it keeps and grows).
 *   - The refcache_build, refcache_build_in_slot and step_attention calls of
 *     one cache share that workspace and the cache's work counter: issue them
 *     in stream order (one stream, or streams ordered by events), not
 *     concurrently.  Calls for different caches may run concurrently.
 *   - The tcgen05 attention kernel and the merge of split items are
 *     launched as programmatic dependents of the previous kernel on the
 *     stream: they wait for it to complete before they read any of the caller's
 *     tensors or the cached K and V (they may read their own work lists, which
 *     were complete when the cache was created, before that), and they
 *     allow the kernel after them to start early.  The cache write of
 *     refcache_build, launched behind the prefill in the same way, overlaps its
 *     tail: it starts once every block of the prefill runs, and so has waited,
 *     and ends after it.  A caller's kernel launched
 *     with programmatic stream serialization after a library call must
 *     therefore wait for its grid dependencies (griddepcontrol.wait) before it
 *     reads the library's outputs; ordinary launches need nothing.
 *   - refcache_build, refcache_build_in_slot and step_attention only launch
 *     kernels (no allocation, no copy), so they can be captured in a CUDA graph and replayed, once a
 *     first call on the device has run outside the capture (the kernels'
 *     attributes are set on first use).  full_attention is not capturable
 *     (it may copy its work list from host memory).
 */
#ifndef REFCACHE_H
#define REFCACHE_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define REFCACHE_API __attribute__((visibility("default")))
#else
#define REFCACHE_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ------------------------------------------------------ */
#define REFCACHE_OK 0
#define REFCACHE_ERR_INVALID_ARG (-1) /* null/misaligned pointer, bad sizes or offsets */
#define REFCACHE_ERR_UNSUPPORTED (-2) /* head_dim not 64/128, no sm_103 device */
#define REFCACHE_ERR_NOT_BUILT (-3)   /* step_attention on a layer whose cache was not built */
#define REFCACHE_ERR_CUDA (-4)        /* a CUDA runtime/driver call failed */
#define REFCACHE_ERR_OOM (-5)         /* device allocation failed or given memory too small */
#define REFCACHE_ERR_TIMEOUT (-6)     /* a kernel's bounded wait ran out (see refcache_status) */

/* ---- mask modes (who the static rows and the live rows attend) ---------- */
/* Sec. 3.3: ST <-> R both ways, live rows attend [LT, X_t, R], not ST.      */
#define REFCACHE_MASK_BEYOND 0
/* Alternative anchor reading: ST rows attend only ST, R rows attend [ST, R],
 * live rows attend [LT, X_t, ST, R]; the cache then keeps ST's K/V too.     */
#define REFCACHE_MASK_BEYOND_ALT 1
/* Sec. 4.1 isolated cache (prior-art topology): R attends only R; every
 * request must have zero anchors.                                            */
#define REFCACHE_MASK_ISOLATED 2

/* Cache format flag, OR-ed into mask_mode of refcache_bytes/refcache_create.
 * An explicitly approximate variant of the paper's exact cache (Sec. 3.3
 * reuses the cached K/V exactly): the cached rows are stored as OCP FP8 E4M3
 * codes with one fp32 scale per (128-row tile of one request, head):
 *   amax = max |x| over the tile's rows and the head's 128 columns,
 *   s = amax / 448, code = E4M3(x * (448 / amax)) (round to nearest even,
 *   IEEE fp32 divide and multiply; code 0 and s = 0 when amax = 0).
 * Layout of one layer (refcache_fp8_ptr): K codes [rows_pad, H, 128], V codes
 * transposed per head [H, 128, rows_pad], scales float32 [rows_pad / 128, H, 4]
 * = (s_K, s_V, log2 s_V, 1 / s_V) (the last two 0 when s_V = 0); each
 * request's cached rows start on a 128-row boundary and pad rows hold code 0.  head_dim must be 128 and the tcgen05 kernel selected.
 * step_attention then quantises each live query row per head the same way
 * (one scale per row), attends the cached keys on E4M3 tensor-core MMAs with
 * E4M3 softmax weights, and the live keys exactly as in the bf16 cache; the
 * prefill (refcache_build's outputs) is unchanged.  Half the cache bytes. */
#define REFCACHE_CACHE_FP8 0x100

/* Kernel selection (refcache_set_kernel): the tcgen05/TMEM/TMA kernel is the
 * default (on CTA pairs with 192-key tiles for the bf16 cache, at both head
 * dims); the mma.sync kernel is the recompiled legacy-tensor-core baseline;
 * TCGEN05_K128 is the same tcgen05 pair kernel with 128-key tiles, kept as a
 * comparison point (the E4M3 cache always uses 128-key tiles). */
#define REFCACHE_KERNEL_TCGEN05 0
#define REFCACHE_KERNEL_MMA_SYNC 1
#define REFCACHE_KERNEL_TCGEN05_K128 2

/*
 * Segment table of a batch of requests (Eq. 1 layout, Sec. 3.3 order).
 * All arrays are HOST memory.
 *   cu_live[batch+1]   offsets of each request's [LT; X_t] rows in the step
 *                      tensors (cu_seqlens style, cu_live[0] = 0, non-decreasing)
 *   cu_static[batch+1] offsets of each request's [ST; R] rows in the prefill
 *                      tensors
 *   n_anchor[batch]    N_ST: the first n_anchor[b] rows of request b's static
 *                      segment are anchors, the rest are R (N_R >= 0)
 *   n_instr[batch]     N_LT (may be NULL): the first rows of each live segment
 *                      are instruction text; LT and X_t are attended alike, so
 *                      it is informational
 */
typedef struct {
  int32_t batch;
  int32_t num_heads;
  int32_t head_dim;
  const int32_t* cu_live;
  const int32_t* cu_static;
  const int32_t* n_anchor;
  const int32_t* n_instr;
} refcache_segments_t;

typedef struct refcache refcache_t; /* opaque; owns the per-layer K/V slots */

/*
 * Device bytes a cache needs for `num_layers` layers (Sec. 3.3: per layer the
 * R rows' K and V, bf16, [cache_rows, num_heads, head_dim] each, plus the
 * anchors' rows in REFCACHE_MASK_BEYOND_ALT; with REFCACHE_CACHE_FP8 the E4M3
 * layout above), plus its small work tables.  Returns 0 for invalid arguments.
 */
REFCACHE_API size_t refcache_bytes(int num_layers, int mask_mode, const refcache_segments_t* seg);

/*
 * Create a cache.  If dev_mem is NULL the library allocates refcache_bytes()
 * with cudaMalloc on the current device and frees it in refcache_destroy;
 * otherwise it uses dev_mem (>= refcache_bytes(), 256-byte aligned, owned by
 * the caller, not freed).  Synchronous.  *out is set only on success.
 *
 * It also plans, for the current device, the per-item work
 * lists of the prefill and the step, (query tile, head) items longest first;
 * a launch hands them out in that order to whichever CTA pair is free,
 * through a work counter kept in the cache's memory (reset by the launch
 * itself when it ends), so the pair that computes an item varies but its
 * arithmetic does not.  full_attention does the same with a counter kept
 * beside its work list; full_attention_noalloc takes items in a fixed order
 * (the same results, bit for bit).  When the step's
 * items do not fill the last round of the GPU's CTA pairs evenly and it ends the
 * step sooner, the items of that round are split by key range into 2-8 parts whose
 * outputs a combine kernel merges.  These lists and an fp32 workspace for the parts (parts x 256
 * rows x (head_dim + 1) x 4 bytes, e.g. 27 MB at 1024^2 with five references)
 * are one more cudaMalloc, freed by refcache_destroy.  Which step items are split depends on the whole
 * batch and the device, so a step output's last bits may differ between
 * batches (never by more than the rounding of a split).  The prefill is never
 * split: refcache_build's outputs and cache bytes for a request depend only on
 * that request's own inputs, whatever else is in the batch and on any GPU.
 */
REFCACHE_API int refcache_create(refcache_t** out, int num_layers, int mask_mode, const refcache_segments_t* seg,
                    void* dev_mem, size_t dev_bytes);

/* Free the cache (waits for the device to finish using it).  NULL is a no-op. */
REFCACHE_API void refcache_destroy(refcache_t* cache);

/*
 * Device pointers of layer `layer`'s K and V slots, each a THD bf16 tensor of
 * *rows rows: request b's cached rows follow request b-1's.  Cached rows are
 * R (Eq. 2), or [ST; R] in REFCACHE_MASK_BEYOND_ALT.  Any output may be NULL.
 * REFCACHE_ERR_UNSUPPORTED for an E4M3 cache.
 */
REFCACHE_API int refcache_kv_ptr(refcache_t* cache, int layer, void** k_slot, void** v_slot, int64_t* rows);

/*
 * Device pointers of layer `layer` of an E4M3 cache (REFCACHE_CACHE_FP8): the
 * K codes [rows_pad, H, 128] (uint8), the V codes [H, 128, rows_pad] (uint8)
 * and the scales [rows_pad / 128, H, 4] (float32), owned by the cache.  Any
 * output may be NULL.  REFCACHE_ERR_UNSUPPORTED for a bf16 cache.
 */
REFCACHE_API int refcache_fp8_ptr(refcache_t* cache, int layer, void** k8, void** vt8, void** scales,
                                  int64_t* rows_pad);

/* 1 if `layer` has been built, 0 if not, < 0 on error. */
REFCACHE_API int refcache_layer_built(refcache_t* cache, int layer);

/*
 * Number of kernels one refcache_build (call = 0), step_attention (call = 1)
 * or refcache_build_in_slot (call = 2) on this cache launches with the kernel
 * family currently selected (refcache_set_kernel): the attention kernel, the
 * cache write (refcache_build, when there are cached rows: a copy, or the
 * E4M3 quantisation) and the combine of split items (step_attention, when the
 * cache's work list has any).  < 0 on error.
 */
REFCACHE_API int refcache_call_launches(refcache_t* cache, int call);

/*
 * Static prefill of one layer (Sec. 3.3; cost (N_R + N_ST)^2 per head,
 * Eq. cost-pre).  q_static/k_static/v_static: [cu_static[batch], H, d] bf16,
 * each request's [ST; R] rows.  Writes o_static (same shape) for every ST and
 * R row, lse_static if non-NULL, and copies the cached rows' K and V into the
 * layer's slots (an E4M3 cache: quantises them).  The result does not depend
 * on any live input, and repeated builds with the same inputs produce the
 * same bytes.
 */
REFCACHE_API int refcache_build(refcache_t* cache, int layer, const void* q_static, const void* k_static,
                   const void* v_static, void* o_static, float* lse_static, float softmax_scale,
                   void* stream);

/*
 * The static prefill of one layer for a caller that projects the cached rows'
 * K and V straight into the cache (the zero-copy path of Sec. 3.3: only R's
 * K/V are kept, so they may be written where they are kept): before the call
 * the layer's slots (refcache_kv_ptr) must hold the cached rows' K and V --
 * R, or [ST; R] in REFCACHE_MASK_BEYOND_ALT -- of every request, in the
 * slot's row order.  Computes what refcache_build computes (rows [ST; R] over
 * keys [ST; R] under the cache's mask mode) and marks the layer built, but
 * reads R's keys and values from the slots and launches no cache write.
 *   q_static: [cu_static[batch], H, d] bf16, each request's [ST; R] queries.
 *   k_anchor, v_anchor: [sum n_anchor, H, d] bf16, the anchors' K and V,
 *     request b's n_anchor[b] rows after request b-1's; NULL when there are
 *     no anchor rows, and ignored (may be NULL) in REFCACHE_MASK_BEYOND_ALT,
 *     whose slots hold the anchors too.
 *   o_static / lse_static as in refcache_build.
 * The keys are tiled from the anchors and from R separately, so the outputs
 * equal refcache_build's up to the rounding order of the sums, and repeated
 * calls on the same inputs give the same bytes.  The slots are only read.
 * REFCACHE_ERR_UNSUPPORTED for an E4M3 cache (REFCACHE_CACHE_FP8), which
 * refcache_build writes from bf16 K and V.
 */
REFCACHE_API int refcache_build_in_slot(refcache_t* cache, int layer, const void* q_static, const void* k_anchor,
                                        const void* v_anchor, void* o_static, float* lse_static, float softmax_scale,
                                        void* stream);

/*
 * One denoising step of one layer (App. C: [LT, X_t] queries over
 * [LT, X_t, R]; cost S (N_R + S) per head, Eq. cost-step).  q_live, k_live,
 * v_live: [cu_live[batch], H, d] bf16, each request's [LT; X_t] rows.  Keys
 * are the request's own live rows followed by its cached rows of `layer`.
 * Writes o_live (same shape) and lse_live if non-NULL.
 * Returns REFCACHE_ERR_NOT_BUILT if the layer was never built, and
 * REFCACHE_ERR_UNSUPPORTED for an E4M3 cache while the mma.sync kernel is
 * selected.
 */
REFCACHE_API int step_attention(refcache_t* cache, int layer, const void* q_live, const void* k_live,
                   const void* v_live, void* o_live, float* lse_live, float softmax_scale,
                   void* stream);

/*
 * Full attention (Sec. 3.2; C_full = T (N_R + S)^2 over T steps, App. C):
 * every row of request b attends every key of request b.  cu_seqlens is a
 * HOST array [batch+1]; q, k, v, o are [cu_seqlens[batch], H, d] bf16.
 * Uses (and on first use or growth allocates) a per-device work-list buffer
 * kept by the library; calls on one device must be ordered on one stream.
 */
REFCACHE_API int full_attention(int batch, int num_heads, int head_dim, const int32_t* cu_seqlens, const void* q,
                   const void* k, const void* v, void* o, float* lse, float softmax_scale,
                   void* stream);

/*
 * full_attention for callers that cannot allocate device memory -- e.g. code
 * running under a custom or pooled allocator that forbids cudaMalloc, or a
 * host runtime that must not grow GPU memory after start-up.  The paper has
 * no counterpart; this is a deployment variant of full_attention above.
 *
 * Same arguments, semantics and results as full_attention, but the work list
 * lives in a fixed array in the library's static device memory (held by every
 * GPU that loads the library until the process exits), so the call allocates
 * nothing: no cudaMalloc, no cudaFree, no allocating library routine.  The
 * caller still passes (and owns) q, k, v, o and lse.
 *   - The array holds REFCACHE_NOALLOC_MAX_TASKS work items (512 KiB).  One
 *     item covers up to 256 query rows of a request (either head_dim), so a
 *     request of n rows needs ceil(n / 256) items: at most 16384 x 256 rows
 *     per call (fewer when requests end mid-item).  Larger inputs are
 *     rejected with REFCACHE_ERR_INVALID_ARG and a message naming the limit.
 *   - The first call on each device looks up the array's device address with
 *     that device current (a one-time set-up).
 *   - Every call rewrites the whole work list it uses, so no state carries
 *     over, but all calls share the one array: calls whose kernels overlap on
 *     the GPU (different streams, or other threads) race.  Order them on one
 *     stream.
 */
#define REFCACHE_NOALLOC_MAX_TASKS 16384
REFCACHE_API int full_attention_noalloc(int batch, int num_heads, int head_dim, const int32_t* cu_seqlens,
                                        const void* q, const void* k, const void* v, void* o, float* lse,
                                        float softmax_scale, void* stream);

/* ---- gradients of the attention calls -------------------------------------
 *
 * With P = exp(scale Q K^T - lse), recomputed from the log-sum-exp that the
 * forward call wrote:
 *   dV = P^T dO, dP = dO V^T, dS = P (dP - rowsum(dO O)), dQ = scale dS K,
 *   dK = scale dS^T Q
 * over exactly the pairs that the forward call attends.  Shared conventions:
 *   - q, k, v, o, lse: inputs and outputs of the forward call; d_o: the gradient
 *     of o.  dq, dk, dv are written (not added to).  All bf16, like the forward
 *     call's tensors, except lse (fp32 [rows, H], not optional here).
 *   - Scores, P, dP, dS and all sums are fp32; P and dS are rounded to bf16 as
 *     operands of their products, gradients once when they are written.
 *   - Every sum has one place and one order: the same inputs give the same bits,
 *     and a request's gradients do not depend on the rest of the batch.
 *   - work: refcache_backward_bytes(rows, H) bytes of device memory, 16-byte
 *     aligned, overwritten; free again when the call's work on the stream is done.
 *   - Every q, k, v, o, d_o row must hold finite values, as in the forward calls.
 *   - They launch kernels only (one over the outputs, then two for every 32
 *     requests) and allocate nothing, so they can be captured in a CUDA graph,
 *     after a first call on the device outside the capture.  Calls share no
 *     state but what the caller passes: they may overlap on several streams,
 *     each with its own work and outputs.
 *   - Outputs must not overlap inputs.
 */
REFCACHE_API size_t refcache_backward_bytes(int64_t rows, int num_heads);

/*
 * Gradient of step_attention: rows = cu_live[batch].  dk_live, dv_live are the
 * gradients of the live rows' own keys; dk_ref, dv_ref [cached rows, H, d] bf16
 * (the slots' row order, refcache_kv_ptr) those of the cached rows, or both NULL
 * when the cache takes no gradient (their work is then left out).  With
 * accumulate != 0 the call adds to what dk_ref and dv_ref hold: several denoising
 * steps of one rollout share a cache.  In bf16 that sum is rounded at each call, n
 * times for n steps, and loses what is below 2^-9 of it; step_attention_backward_ref_f32
 * holds it in fp32.
 * A bf16 cache; REFCACHE_ERR_UNSUPPORTED for an E4M3 cache, whose quantisation has
 * no gradient, REFCACHE_ERR_NOT_BUILT for a layer that was never built.
 */
REFCACHE_API int step_attention_backward(refcache_t* cache, int layer, const void* q_live, const void* k_live,
                                         const void* v_live, const void* o_live, const float* lse_live,
                                         const void* do_live, void* dq_live, void* dk_live, void* dv_live, void* dk_ref,
                                         void* dv_ref, int accumulate, void* work, float softmax_scale, void* stream);

/* The same with dk_ref and dv_ref in fp32. */
REFCACHE_API int step_attention_backward_ref_f32(refcache_t* cache, int layer, const void* q_live, const void* k_live,
                                                 const void* v_live, const void* o_live, const float* lse_live,
                                                 const void* do_live, void* dq_live, void* dk_live, void* dv_live,
                                                 float* dk_ref, float* dv_ref, int accumulate, void* work,
                                                 float softmax_scale, void* stream);

/*
 * Gradient of refcache_build: rows = cu_static[batch], under the cache's mask
 * mode.  dk_ref, dv_ref (NULL, or [cached rows, H, d] bf16 from
 * step_attention_backward) are added to the cached rows' gradients before they
 * are rounded: the cached K and V are the static rows' own.  Reads no slot of the
 * cache (`layer` is only checked), so the layer may have been rebuilt since.
 */
REFCACHE_API int refcache_build_backward(refcache_t* cache, int layer, const void* q_static, const void* k_static,
                                         const void* v_static, const void* o_static, const float* lse_static,
                                         const void* do_static, void* dq_static, void* dk_static, void* dv_static,
                                         const void* dk_ref, const void* dv_ref, void* work, float softmax_scale,
                                         void* stream);

/* The same with dk_ref and dv_ref in fp32. */
REFCACHE_API int refcache_build_backward_ref_f32(refcache_t* cache, int layer, const void* q_static, const void* k_static,
                                                 const void* v_static, const void* o_static, const float* lse_static,
                                                 const void* do_static, void* dq_static, void* dk_static, void* dv_static,
                                                 const float* dk_ref, const float* dv_ref, void* work,
                                                 float softmax_scale, void* stream);

/* Gradient of full_attention (and full_attention_noalloc); capturable, allocates nothing. */
REFCACHE_API int full_attention_backward(int batch, int num_heads, int head_dim, const int32_t* cu_seqlens,
                                         const void* q, const void* k, const void* v, const void* o, const float* lse,
                                         const void* d_o, void* dq, void* dk, void* dv, void* work, float softmax_scale,
                                         void* stream);

/* ---- from a projection to the attention's q, k and v ----------------------
 *
 * Per head RMS norm of query and key and rotary positions with several axes
 * (frame, height and width of image tokens, for instance):
 *   n = x / sqrt(mean(x^2) + eps) * weight        (weight NULL: n = x)
 *   (a, b) -> (a cos t - b sin t, a sin t + b cos t) for each pair of n,
 *   t = position[axis of the pair] * theta^(-2 j / axis_dim), j = its number on the axis
 * Axis i takes the next axis_dims[i] / 2 pairs; pairs past the axes' dims (their
 * sum may be below head_dim) are not turned.  Pair j is elements (2 j, 2 j + 1)
 * when interleaved, else (j, j + head_dim / 2).  Arithmetic in fp32, angles exact
 * for positions up to 2^24 in magnitude, one rounding to bf16 at the end.
 */
#define REFCACHE_ROPE_MAX_AXES 4
typedef struct {
  int32_t head_dim, num_axes, interleaved;
  float turn_hi[64], turn_lo[64]; /* frequency / (2 pi) of each pair, as a sum of two */
  uint8_t axis[64];               /* axis of each pair */
} refcache_rope_t;

/* Fill *rope (host memory, the caller's; needs no device). */
REFCACHE_API int refcache_rope_init(refcache_rope_t* rope, int head_dim, int num_axes, const int32_t* axis_dims,
                                    double theta, int interleaved);

/* The rows of one call.  positions, row_map and the weights are device memory. */
typedef struct {
  int64_t rows;              /* token rows of q, k and v */
  int64_t out_rows;          /* rows of q_out, k_out and v_out */
  int32_t num_heads;
  int32_t weight_f32;        /* weights fp32 (else bf16) */
  const int32_t* positions;  /* [rows, num_axes] */
  const int32_t* row_map;    /* row i goes to row row_map[i] of the outputs (distinct; outside
                                [0, out_rows): dropped, its gradient is 0); NULL: to row i */
  const void* weight_q;      /* [head_dim], or NULL: not normalised */
  const void* weight_k;
  float eps;
} refcache_rope_rows_t;

/*
 * q, k, v: rows of num_heads x head_dim bf16, contiguous within a row, ld elements
 * between rows (a multiple of 8: a fused projection's [rows, 3, H, d] may be passed
 * as three tensors).  Outputs must not overlap inputs; they are [out_rows, H, d]
 * bf16, packed, as the attention calls take them; k_out and v_out may be a cache's slots (refcache_kv_ptr), before
 * refcache_build_in_slot.  v is moved only.  Each of the three may be NULL together
 * with its output.  Output rows that no row goes to are left as they are.
 */
REFCACHE_API int refcache_qkv_rope(const refcache_rope_t* rope, const refcache_rope_rows_t* rows, const void* q,
                                   int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v, void* q_out,
                                   void* k_out, void* v_out, void* stream);

/*
 * Its gradient: from those of the outputs ([out_rows, H, d] packed) to dq, dk, dv
 * (rows with ld elements between them) and the weights' (fp32 [head_dim], may be
 * NULL).  q and k are the forward call's inputs, read where they were normalised.
 * work: refcache_qkv_rope_backward_bytes bytes of device memory, needed with a
 * weight.  The weights' sums are taken in a fixed order.
 */
REFCACHE_API size_t refcache_qkv_rope_backward_bytes(const refcache_rope_t* rope);
REFCACHE_API int refcache_qkv_rope_backward(const refcache_rope_t* rope, const refcache_rope_rows_t* rows, const void* q,
                                            int64_t ld_q, const void* k, int64_t ld_k, const void* dq_out,
                                            const void* dk_out, const void* dv_out, void* dq, int64_t ld_dq, void* dk,
                                            int64_t ld_dk, void* dv, int64_t ld_dv, float* dweight_q, float* dweight_k,
                                            void* work, void* stream);

/* ---- gated residual and norm ----------------------------------------------
 *
 * The end of one half of a transformer block and the start of the next, for rows
 * of `width` bf16 (a multiple of 8, at most 8192), packed, requests back to back:
 *   h = branch, or post_norm(branch) * post_weight
 *   x_out = x + gate * h                            (no branch: x)
 *   y = norm(x_out) * weight * (1 + scale) + shift  (before x_out is rounded)
 * gate, scale and shift are rows of the request (ld elements between requests'
 * rows, a multiple of 8; 0: one row for all requests); gate NULL is 1, scale and
 * shift NULL are 0, weights NULL are 1.
 * Layer norm: (x - mean) / sqrt(var + eps); RMS norm: x / sqrt(mean(x^2) +
 * eps).  Statistics and arithmetic in fp32.
 */
#define REFCACHE_NORM_NONE 0
#define REFCACHE_NORM_LAYER 1
#define REFCACHE_NORM_RMS 2
typedef struct {
  int32_t batch;
  int32_t width;
  const int32_t* cu_rows;   /* HOST [batch + 1]: first row of each request, cu_rows[0] = 0 */
  int32_t norm, post_norm;  /* REFCACHE_NORM_* */
  int32_t mod_f32;          /* gate, scale, shift and the weights are fp32 (else bf16) */
  float eps;
  const void *gate, *scale, *shift; /* device, [batch, width] with ld_* */
  int64_t ld_gate, ld_scale, ld_shift;
  const void *weight, *post_weight; /* device, [width] */
} refcache_gated_norm_t;

/*
 * x, branch (may be NULL): [rows, width] bf16.  x_out (may be NULL, or x itself) and
 * y (may be NULL) are written; they overlap nothing else.
 */
REFCACHE_API int refcache_gated_norm(const refcache_gated_norm_t* p, const void* x, const void* branch, void* x_out,
                                     void* y, void* stream);

/*
 * Its gradient.  x_out: the forward call's output (its x where there is no
 * branch), needed with dy; dy, dx_out: gradients of y and x_out, either may be
 * NULL for zero, not both.  Written, each unless NULL: dx, d_branch [rows, width] bf16;
 * d_gate, d_scale, d_shift fp32 [batch, width]; d_weight, d_post_weight fp32 [width].
 * A request without rows has gradients of zero and adds nothing to the weights', whatever
 * its gate and scale hold; without any rows all tensors of rows may be NULL.
 * The statistics are found again from x_out and branch.  Column sums are fp32, in a
 * fixed order for a given device.  work: refcache_gated_norm_backward_bytes(p)
 * bytes of device memory, 16-byte aligned.
 */
REFCACHE_API size_t refcache_gated_norm_backward_bytes(const refcache_gated_norm_t* p);
REFCACHE_API int refcache_gated_norm_backward(const refcache_gated_norm_t* p, const void* x_out, const void* branch,
                                              const void* dy, const void* dx_out, void* dx, void* d_branch, float* d_gate,
                                              float* d_scale, float* d_shift, float* d_weight, float* d_post_weight,
                                              void* work, void* stream);

/* ---- clipping of gradients --------------------------------------------------
 *
 * norm = sqrt(sum of squares of all n tensors), out_i = grads_i * min(1, max_norm /
 * (norm + 1e-6)).  The lists are HOST arrays: device pointers, element counts, and
 * types[i] = REFCACHE_CLIP_* flags.  Tensors need the alignment of their elements
 * only.  out NULL: in place (nothing is written where the factor is 1).  norm: device
 * fp32, may be NULL.  max_norm may be +inf: the norm alone, with out = grads whatever it
 * is.  Under a finite bound a norm that is NaN makes the outputs NaN, and an infinite
 * one makes finite elements 0.  (Squares are summed
 * in fp32 per thread and in fp64 from there on: the norm is infinite where a
 * thread's squares overflow fp32, and squares below its range count as 0.)  work: refcache_clip_gradients_bytes(n) bytes of
 * device memory, 16-byte aligned.
 */
#define REFCACHE_CLIP_GRAD_F32 1 /* gradient fp32 (else bf16) */
#define REFCACHE_CLIP_OUT_F32 2  /* output fp32 (else bf16) */
REFCACHE_API size_t refcache_clip_gradients_bytes(int n);
REFCACHE_API int refcache_clip_gradients(int n, const void* const* grads, void* const* out, const int64_t* counts,
                                         const int32_t* types, float max_norm, float* norm, void* work, void* stream);

/* ---- linear layers in 8 bits ----------------------------------------------
 *
 * The 8-bit form of rows (bf16 activations or gradients) is OCP E4M3 codes and, for
 * each block of 128 columns of a row, a power of two as scale, kept as UE8M0: byte b
 * is 2^(b - 127), the smallest with amax / 2^(b - 127) <= 448 (127 for a block of
 * zeros, at least 1); code = E4M3(x / 2^(b - 127)), round to nearest even.  A block
 * that holds a NaN or an infinity has b = 255 and NaN codes: all of it is NaN.  A
 * weight has one scale for each 128 x 128.  Where a row's last block is short it is
 * over the columns that are there.
 *
 * Rows in this form are what the products below take, and serve as the checkpoint of
 * the activations until the backward pass, which reads them as they are.
 *   - Widths are multiples of 16 up to 2^20, rows up to 2^31 - 513.
 *   - Codes are packed [rows, width], 16-byte aligned; scales are rows of
 *     REFCACHE_F8_PITCH(width) bytes, 16-byte aligned, of which the first
 *     ceil(width / 128) count.
 *   - tiles, REFCACHE_F8_TILES(rows, width) bytes, 16-byte aligned, hold the same scales once
 *     more, as the tensor cores take them: the four bytes of 512 columns of row r are the word at
 *     512 (g ceil(rows / 128) + r / 128) + 16 (r % 32) + 4 (r / 32 % 4) for the g-th 512
 *     columns.  A weight's block has its byte for all of its 128 rows, those behind the weight's
 *     last one too.  What else belongs to no row or block may hold anything, before and after a call.
 *   - Products are summed in fp32 by the tensor cores, whose additions cut off what does not fit: y is off by up to 3e-7 of its norm at
 *     4096 columns of x and 1.5e-6 from 16384 on where the products' signs vary, by 2e-6 and 1.2e-5 (toward zero) where they are all alike, dw
 *     by up to 1e-6 at 20608 rows.  Results are rounded once; a code or a scale next to a border may be its neighbour.
 *   - bf16 tensors of rows may have ld elements between rows (a multiple of 8).
 *   - Outputs, and weight_grad's work, that overlap inputs or each other are refused (but for dw over add; of
 *     rows that lie apart only the first one is looked at).
 *   - The calls launch kernels only and allocate nothing: they can be captured in a
 *     CUDA graph, after a first call on the device outside the capture, and may overlap
 *     on several streams.  Sums have a fixed order for a given device: the same inputs
 *     give the same bits.
 */
#define REFCACHE_F8_PITCH(width) (((width) + 511) / 512 * 4)
#define REFCACHE_F8_TILES(rows, width) (((width) + 511) / 512 * (((int64_t)(rows) + 127) / 128) * 512)
typedef struct {
  int64_t rows;
  int32_t width;
  void* codes;  /* [rows, width] */
  void* scales; /* [rows, REFCACHE_F8_PITCH(width)] */
  void* tiles;  /* REFCACHE_F8_TILES(rows, width) bytes */
} refcache_f8_rows_t;
typedef struct {
  int32_t out_width, in_width; /* w is [out_width, in_width] */
  void *codes, *scales;        /* [out, in]; [ceil(out / 128), REFCACHE_F8_PITCH(in)] */
  void* tiles;                 /* REFCACHE_F8_TILES(out, in) */
  void *codes_t, *scales_t;    /* transposed: [in, out]; [ceil(in / 128), REFCACHE_F8_PITCH(out)] (same values) */
  void* tiles_t;               /* REFCACHE_F8_TILES(in, out) */
} refcache_f8_weight_t;

/* x: [out->rows, out->width] bf16, ld elements between rows. */
REFCACHE_API int refcache_f8_quantize(const void* x, int64_t ld, const refcache_f8_rows_t* out, void* stream);

/* w: [out_width, in_width], packed, fp32 (w_f32 != 0) or bf16.  codes_t, scales_t and tiles_t may all be NULL. */
REFCACHE_API int refcache_f8_quantize_weight(const void* w, int w_f32, const refcache_f8_weight_t* out, void* stream);

/*
 * y = x w^T + bias [rows, out_width] (reads codes and tiles), or with transposed != 0
 * y = x w [rows, in_width] (codes_t, tiles_t): a layer's output, and its input's
 * gradient from the 8-bit form of its output's.  y bf16; bias: one value for each
 * column of y, fp32 (bias_f32 != 0) or bf16, or NULL.
 */
REFCACHE_API int refcache_f8_linear(const refcache_f8_rows_t* x, const refcache_f8_weight_t* w, int transposed, const void* bias,
                                    int bias_f32, void* y, int64_t ld_y, void* stream);

/*
 * An MLP's first layer: u = x w^T + bias, a = the 8-bit form of gelu(u), u8 (may be
 * NULL) that of u, the checkpoint for the gradient.  u is not rounded before it goes into
 * either.  form: the normal distribution's function, or its tanh approximation.
 */
#define REFCACHE_GELU_ERF 0
#define REFCACHE_GELU_TANH 1
REFCACHE_API int refcache_f8_linear_gelu(const refcache_f8_rows_t* x, const refcache_f8_weight_t* w, const void* bias, int bias_f32,
                                         int form, const refcache_f8_rows_t* a, const refcache_f8_rows_t* u8, void* stream);

/*
 * Its gradient together with that of the layer behind it: from the 8-bit form of dy, the
 * gradient of that layer's output, and its weight w (reads codes_t, tiles_t),
 * du = (dy w) gelu'(u) with u as u8 holds it.  du [rows, in_width of w] bf16 and du8, the 8-bit
 * form of du before its rounding, are written; either may be NULL, not both.
 */
REFCACHE_API int refcache_f8_linear_gelu_backward(const refcache_f8_rows_t* dy, const refcache_f8_weight_t* w, int form,
                                                  const refcache_f8_rows_t* u8, void* du, int64_t ld_du,
                                                  const refcache_f8_rows_t* du8, void* stream);

/*
 * The weight's gradient: dw = add + dy^T x [out_width, width of x], fp32 (dw_f32 != 0) or
 * bf16, packed; add like dw, dw itself or NULL; d_bias = sums of dy over the rows, fp32
 * [out_width], or NULL.  dy [rows of x, out_width] bf16.  x's values are taken as they
 * are (exact in bf16 from 2^-126 on; 2^128, to which the largest bf16 values round, as 255 * 2^120): the
 * product is bf16 with fp32 sums.  Without rows dw is add, or zero.
 * work: refcache_f8_weight_grad_bytes bytes of device memory (x's values in bf16, at most 256 MB of them
 * or 256 columns at a time, and partial sums where dw is small), 16-byte aligned; may be NULL without rows.
 */
REFCACHE_API size_t refcache_f8_weight_grad_bytes(int64_t rows, int out_width, int in_width);
REFCACHE_API int refcache_f8_weight_grad(const void* dy, int64_t ld_dy, const refcache_f8_rows_t* x, int out_width, const void* add,
                                         void* dw, int dw_f32, float* d_bias, void* work, void* stream);

/*
 * Synchronise `stream`, then read and clear the current device's error word
 * written by kernels whose bounded waits ran out.  Returns REFCACHE_OK,
 * REFCACHE_ERR_TIMEOUT or REFCACHE_ERR_CUDA.
 * The word is one per device: every kernel of this library on the device (any
 * cache, any stream, full_attention too) writes it, and the first
 * refcache_status call that reads it clears it.  To learn which cache's launch
 * gave up, use refcache_cache_status.
 */
REFCACHE_API int refcache_status(void* stream);

/*
 * The same for one cache: synchronise `stream`, then read and clear the error
 * word of `cache`, which the kernels launched by refcache_build,
 * refcache_build_in_slot and step_attention on this cache set (besides the
 * device word) when a bounded wait runs out.  Returns REFCACHE_OK,
 * REFCACHE_ERR_TIMEOUT, REFCACHE_ERR_INVALID_ARG (NULL cache, or the current
 * device is not the cache's) or REFCACHE_ERR_CUDA.  It clears only this
 * cache's word, and refcache_status only the device word.
 */
REFCACHE_API int refcache_cache_status(refcache_t* cache, void* stream);

/*
 * Wait limit of every in-kernel wait, nanoseconds (default 1e9; less than REFCACHE_LEAST_WAIT_NS counts as
 * that).  Returns the old value.  The same limit holds for the waits of a kernel that gives up for its own loads and MMAs
 * in flight, which take microseconds: a shorter one would let it leave before they are done.
 */
#define REFCACHE_LEAST_WAIT_NS 1000000ull
REFCACHE_API uint64_t refcache_set_wait_timeout_ns(uint64_t ns);

/* Select the kernel for subsequent calls (REFCACHE_KERNEL_*); returns the old one or < 0. */
REFCACHE_API int refcache_set_kernel(int kernel);

/*
 * Debug fault injection on the host side of the wait protocol: when `on` is
 * non-zero, the next launch's TMA producer skips its first K-tile load, so
 * the consumers' bounded waits run out and the kernel reports
 * REFCACHE_ERR_TIMEOUT through refcache_status() instead of hanging.  The
 * switch clears itself after one call.  Only the tcgen05 kernels have it.
 *
 * In a gradient call, bits 0-7 are the load before which a producer stops (1: it
 * loads nothing), of the queries kernel, or of the keys kernel with bit 8, in the
 * first CTA of each pair, or in the second with bit 9.  In an 8-bit product, bits 0-7
 * and 9 likewise (products of few rows, whose CTAs are no pairs: in each cluster's CTAs of even or odd number).
 */
REFCACHE_API void refcache_debug_skip_first_load(int on);

/*
 * Diagnostic: the rate of the GPU's exponential unit (ex2.approx.f32, the
 * special-function unit) on the current device, in exponentials per clock per
 * SM (median over the SMs), written to *per_clk_per_sm (host).  The softmax
 * of the attention kernels evaluates one exponential per visible (query, key)
 * pair of one head; this rate gives that work's floor beside the tensor-core
 * roofline.  The paper has no counterpart.  Runs one short kernel (one CTA
 * per SM, about 0.1 ms) on `stream` and synchronises it; allocates nothing.
 * Returns REFCACHE_ERR_INVALID_ARG for a NULL pointer.
 */
REFCACHE_API int refcache_ex2_rate(double* per_clk_per_sm, void* stream);

/* Copy the calling thread's last error message into buf (NUL-terminated); returns its length. */
REFCACHE_API int refcache_last_error(char* buf, size_t n);

/* Library version string. */
REFCACHE_API const char* refcache_version(void);

#ifdef __cplusplus
}
#endif

#endif /* REFCACHE_H */
