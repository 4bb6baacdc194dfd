"""Thin ctypes binding of librefcache.so (include/refcache.h).

Argument marshalling only: torch tensors are passed as raw device pointers,
the current torch stream as the CUDA stream.  A call's tensors are on one device,
the cache's or else the current one.  Every attention step runs in the
library's CUDA kernels; when the library is missing this module raises, it
never falls back to another implementation.
"""
from __future__ import annotations

import ctypes
import math
import os
from array import array
from typing import Optional, Sequence

from . import build as _build

OK = 0
ERR_INVALID_ARG = -1
ERR_UNSUPPORTED = -2
ERR_NOT_BUILT = -3
ERR_CUDA = -4
ERR_OOM = -5
ERR_TIMEOUT = -6

MASK_MODES = {"beyond": 0, "beyond_alt": 1, "isolated": 2}
KERNELS = {"tcgen05": 0, "mma_sync": 1, "tcgen05_k128": 2}
NORMS = {None: 0, "layer": 1, "rms": 2}
ROPE_PAIRS = {"halves": 0, "interleaved": 1}
CACHE_DTYPES = {"bf16": 0, "fp8": 0x100}  # REFCACHE_CACHE_FP8: E4M3 codes with per-tile scales

EXPORTED = (
    "refcache_bytes", "refcache_create", "refcache_destroy", "refcache_kv_ptr", "refcache_layer_built",
    "refcache_build", "step_attention", "full_attention", "refcache_status", "refcache_set_wait_timeout_ns",
    "refcache_set_kernel", "refcache_debug_skip_first_load", "refcache_last_error", "refcache_version",
    "full_attention_noalloc", "refcache_call_launches", "refcache_fp8_ptr", "refcache_build_in_slot",
    "refcache_cache_status", "refcache_ex2_rate",
    "refcache_backward_bytes", "step_attention_backward", "refcache_build_backward", "full_attention_backward",
    "step_attention_backward_ref_f32", "refcache_build_backward_ref_f32",
    "refcache_rope_init", "refcache_qkv_rope", "refcache_qkv_rope_backward_bytes", "refcache_qkv_rope_backward",
    "refcache_gated_norm", "refcache_gated_norm_backward_bytes", "refcache_gated_norm_backward",
    "refcache_clip_gradients_bytes", "refcache_clip_gradients",
)
NOALLOC_MAX_TASKS = 16384


class RefCacheError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"refcache error {code}: {msg}")
        self.code = code


class _Segments(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("num_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("cu_live", ctypes.POINTER(ctypes.c_int32)), ("cu_static", ctypes.POINTER(ctypes.c_int32)),
        ("n_anchor", ctypes.POINTER(ctypes.c_int32)), ("n_instr", ctypes.POINTER(ctypes.c_int32)),
    ]


class _Rope(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("num_axes", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("turn_hi", ctypes.c_float * 64), ("turn_lo", ctypes.c_float * 64), ("axis", ctypes.c_uint8 * 64)]


class _RopeRows(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("out_rows", ctypes.c_int64), ("num_heads", ctypes.c_int32),
                ("weight_f32", ctypes.c_int32), ("positions", ctypes.c_void_p), ("row_map", ctypes.c_void_p),
                ("weight_q", ctypes.c_void_p), ("weight_k", ctypes.c_void_p), ("eps", ctypes.c_float)]


class _GatedNorm(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("width", ctypes.c_int32), ("cu_rows", ctypes.POINTER(ctypes.c_int32)),
                ("norm", ctypes.c_int32), ("post_norm", ctypes.c_int32), ("mod_f32", ctypes.c_int32), ("eps", ctypes.c_float),
                ("gate", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("shift", ctypes.c_void_p),
                ("ld_gate", ctypes.c_int64), ("ld_scale", ctypes.c_int64), ("ld_shift", ctypes.c_int64),
                ("weight", ctypes.c_void_p), ("post_weight", ctypes.c_void_p)]


_lib = None


def lib_path() -> str:
    return _build.LIB_PATH


def load(path: Optional[str] = None):
    """Load the CUDA library.  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"CUDA library not built ({path} missing): run __graft_entry__.build() "
                           "or python -m paper_2608_21229_gb300.build")
    L = ctypes.CDLL(path)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
    segp = ctypes.POINTER(_Segments)
    L.refcache_bytes.argtypes = [i32, i32, segp]
    L.refcache_bytes.restype = ctypes.c_size_t
    L.refcache_create.argtypes = [ctypes.POINTER(vp), i32, i32, segp, vp, ctypes.c_size_t]
    L.refcache_destroy.argtypes = [vp]
    L.refcache_destroy.restype = None
    L.refcache_kv_ptr.argtypes = [vp, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(i64)]
    L.refcache_fp8_ptr.argtypes = [vp, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                   ctypes.POINTER(i64)]
    L.refcache_layer_built.argtypes = [vp, i32]
    L.refcache_call_launches.argtypes = [vp, i32]
    L.refcache_build.argtypes = [vp, i32, vp, vp, vp, vp, vp, f32, vp]
    L.refcache_build_in_slot.argtypes = [vp, i32, vp, vp, vp, vp, vp, f32, vp]
    L.step_attention.argtypes = [vp, i32, vp, vp, vp, vp, vp, f32, vp]
    L.full_attention.argtypes = [i32, i32, i32, ctypes.POINTER(ctypes.c_int32), vp, vp, vp, vp, vp, f32, vp]
    L.full_attention_noalloc.argtypes = [i32, i32, i32, ctypes.POINTER(ctypes.c_int32), vp, vp, vp, vp, vp, f32,
                                         vp]
    L.refcache_backward_bytes.argtypes = [i64, i32]
    L.refcache_backward_bytes.restype = ctypes.c_size_t
    L.step_attention_backward.argtypes = [vp, i32] + [vp] * 11 + [i32, vp, f32, vp]
    L.refcache_build_backward.argtypes = [vp, i32] + [vp] * 12 + [f32, vp]
    L.step_attention_backward_ref_f32.argtypes = L.step_attention_backward.argtypes
    L.refcache_build_backward_ref_f32.argtypes = L.refcache_build_backward.argtypes
    L.full_attention_backward.argtypes = [i32, i32, i32, ctypes.POINTER(ctypes.c_int32)] + [vp] * 10 + [f32, vp]
    ropep, rowsp, normp = ctypes.POINTER(_Rope), ctypes.POINTER(_RopeRows), ctypes.POINTER(_GatedNorm)
    L.refcache_rope_init.argtypes = [ropep, i32, i32, ctypes.POINTER(ctypes.c_int32), ctypes.c_double, i32]
    L.refcache_qkv_rope.argtypes = [ropep, rowsp] + [vp, i64] * 3 + [vp] * 4
    L.refcache_qkv_rope_backward_bytes.argtypes = [ropep]
    L.refcache_qkv_rope_backward_bytes.restype = ctypes.c_size_t
    L.refcache_qkv_rope_backward.argtypes = [ropep, rowsp, vp, i64, vp, i64, vp, vp, vp] + [vp, i64] * 3 + [vp] * 4
    L.refcache_gated_norm.argtypes = [normp] + [vp] * 5
    L.refcache_gated_norm_backward_bytes.argtypes = [normp]
    L.refcache_gated_norm_backward_bytes.restype = ctypes.c_size_t
    L.refcache_gated_norm_backward.argtypes = [normp] + [vp] * 13
    L.refcache_clip_gradients_bytes.argtypes = [i32]
    L.refcache_clip_gradients_bytes.restype = ctypes.c_size_t
    L.refcache_clip_gradients.argtypes = [i32, vp, vp, vp, vp, f32, vp, vp, vp]
    L.refcache_status.argtypes = [vp]
    L.refcache_cache_status.argtypes = [vp, vp]
    L.refcache_set_wait_timeout_ns.argtypes = [ctypes.c_uint64]
    L.refcache_set_wait_timeout_ns.restype = ctypes.c_uint64
    L.refcache_set_kernel.argtypes = [i32]
    L.refcache_debug_skip_first_load.argtypes = [i32]
    L.refcache_ex2_rate.argtypes = [ctypes.POINTER(ctypes.c_double), vp]
    L.refcache_debug_skip_first_load.restype = None
    L.refcache_last_error.argtypes = [ctypes.c_char_p, ctypes.c_size_t]
    L.refcache_version.restype = ctypes.c_char_p
    for name in EXPORTED:
        getattr(L, name)
    _lib = L
    return L


def last_error() -> str:
    buf = ctypes.create_string_buffer(1024)
    load().refcache_last_error(buf, len(buf))
    return buf.value.decode(errors="replace")


def _check(code: int):
    if code != OK:
        raise RefCacheError(code, last_error())


def _arr(vals: Optional[Sequence[int]]):
    if vals is None:
        return None
    return (ctypes.c_int32 * len(vals))(*[int(v) for v in vals])


def _device() -> int:
    """The current device, on which calls without a cache launch (-2, no tensor's, where there is none)."""
    global _get_device
    if _get_device is None:
        import torch

        _get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    try:
        return _get_device()
    except (AssertionError, RuntimeError):
        return -2


_get_device = None  # () -> the current device, once torch is in use


def _elsewhere(t, device, name=None):
    """The error of a tensor that is not on the device that the call runs on, whose kernels could not, or not in order, read it."""
    what = "" if name is None else name + ": "
    if not t.is_cuda:
        return ValueError(what + "tensor must live on the GPU")
    return ValueError(f"{what}tensor is on cuda:{t.get_device()}, the call runs on cuda:{device}")


def _ptr(t, device, name=None) -> Optional[int]:
    if t is None:
        return None
    if t.get_device() != device:
        raise _elsewhere(t, device, name)
    if not t.is_contiguous():
        raise ValueError(("" if name is None else name + ": ") + "tensor must be contiguous")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        global _raw_stream
        if _raw_stream is None:
            import torch

            # the handle without a Stream object around it (3 us a call)
            raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device
            _raw_stream = (lambda: raw(device())) if raw else (lambda: torch.cuda.current_stream().cuda_stream)
        return _raw_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


_raw_stream = None  # () -> the current stream's handle, once torch is in use


def _check_thd(name, t, rows, H, D):
    import torch

    if t is None:
        raise ValueError(f"{name} is required")
    if t.dtype != torch.bfloat16 or tuple(t.shape) != (rows, H, D):
        raise ValueError(f"{name}: expected bf16 [{rows}, {H}, {D}], got {t.dtype} {tuple(t.shape)}")


_bf16 = None  # torch.bfloat16, once torch is in use


def _thd_ptrs(named, rows, H, D, device):
    """The device pointers of THD tensors on `device`, which _check_thd and _ptr check in
    this order.  The first line is what a good call runs: the separate checks
    took a third of the 11 us that the host spends on a small step."""
    global _bf16
    if _bf16 is None:
        import torch

        _bf16 = torch.bfloat16
    shape = (rows, H, D)
    for _, t in named:
        if t is None or t.dtype is not _bf16 or t.shape != shape or t.get_device() != device or not t.is_contiguous():
            break
    else:
        return [t.data_ptr() for _, t in named]
    for name, t in named:
        _check_thd(name, t, rows, H, D)
    return [_ptr(t, device, name) for name, t in named]


def set_kernel(name: str) -> str:
    old = load().refcache_set_kernel(KERNELS[name])
    _check(0 if old >= 0 else old)
    return {v: k for k, v in KERNELS.items()}[old]


def set_wait_timeout_ns(ns: int) -> int:
    return int(load().refcache_set_wait_timeout_ns(int(ns)))


def debug_skip_first_load(on: int = 1) -> None:
    load().refcache_debug_skip_first_load(int(on))


def status(stream=None) -> int:
    """Synchronise the stream and return the device error word as a status code."""
    return int(load().refcache_status(_stream(stream)))


def ex2_rate(stream=None) -> float:
    """Exponentials (ex2.approx.f32) per clock per SM measured on the current
    device by the library's probe kernel."""
    v = ctypes.c_double(0.0)
    _check(load().refcache_ex2_rate(ctypes.byref(v), _stream(stream)))
    return float(v.value)


def version() -> str:
    return load().refcache_version().decode()


def default_scale(head_dim: int) -> float:
    return 1.0 / math.sqrt(head_dim)


class Segments:
    """Host segment table (refcache_segments_t)."""

    def __init__(self, num_heads, head_dim, cu_live, cu_static, n_anchor, n_instr=None):
        self.num_heads, self.head_dim = int(num_heads), int(head_dim)
        self.cu_live, self.cu_static = list(cu_live), list(cu_static)
        self.n_anchor = list(n_anchor)
        self.n_instr = None if n_instr is None else list(n_instr)
        self.batch = len(self.n_anchor)
        self._keep = [_arr(self.cu_live), _arr(self.cu_static), _arr(self.n_anchor), _arr(self.n_instr)]
        self.c = _Segments(self.batch, self.num_heads, self.head_dim, *self._keep)

    @classmethod
    def from_workload(cls, w):
        return cls(w.num_heads, w.head_dim, w.cu_live, w.cu_static, w.n_anchor, w.n_instr)

    @property
    def live_rows(self):
        return self.cu_live[-1]

    @property
    def static_rows(self):
        return self.cu_static[-1]


class RefCache:
    """The persistent per-layer reference K/V cache (refcache_t).

    Device memory for the cache comes from torch (one uint8 tensor) and is
    handed to refcache_create, so the library itself allocates nothing.
    """

    _slots = None  # (first byte of layer 0's K slot in the cache memory, rows), once kv() has asked for it

    def __init__(self, seg: Segments, num_layers: int = 1, mask_mode: str = "beyond", device=None,
                 cache_dtype: str = "bf16"):
        import torch

        L = load()
        self.seg, self.num_layers, self.mask_mode = seg, int(num_layers), mask_mode
        self.cache_dtype = cache_dtype
        flags = MASK_MODES[mask_mode] | CACHE_DTYPES[cache_dtype]
        nbytes = L.refcache_bytes(self.num_layers, flags, ctypes.byref(seg.c))
        if nbytes == 0:
            # the planner rejected the arguments: surface its message
            h = ctypes.c_void_p()
            _check(L.refcache_create(ctypes.byref(h), self.num_layers, flags, ctypes.byref(seg.c),
                                     ctypes.c_void_p(1), 0))
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self.mem = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.h = ctypes.c_void_p()
        with torch.cuda.device(device):
            _check(L.refcache_create(ctypes.byref(self.h), self.num_layers, flags, ctypes.byref(seg.c),
                                     ctypes.c_void_p(self.mem.data_ptr()), nbytes))

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            load().refcache_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def kv(self, layer: int):
        """(K slot, V slot) of a layer as bf16 [cache_rows, H, D] views of the cache memory."""
        import torch

        H, D = self.seg.num_heads, self.seg.head_dim
        # The slots of all layers lie one after the other, K before V, so one answer of
        # the library serves every layer (asking takes half the call's time).  The views
        # are made anew each time: one made under inference_mode or no_grad carries that
        # with it and cannot be written to outside.
        if self._slots is None or self.h is None or type(layer) is not int or not 0 <= layer < self.num_layers:
            k, v, rows = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_int64()
            _check(load().refcache_kv_ptr(self.h, layer, ctypes.byref(k), ctypes.byref(v), ctypes.byref(rows)))
            self._slots = (k.value - self.mem.data_ptr() - 4 * layer * rows.value * H * D, rows.value)
        first, rows = self._slots
        n = rows * H * D * 2

        def view(off):
            return self.mem[off:off + n].view(torch.bfloat16).view(rows, H, D)

        off = first + 2 * n * layer
        return view(off), view(off + n)

    def fp8(self, layer: int):
        """E4M3 cache of a layer as views of the cache memory: (K codes uint8
        [rows_pad, H, D], V codes uint8 [H, D, rows_pad], scales float32
        [rows_pad / 128, H, 4] = (s_K, s_V, log2 s_V, 1 / s_V))."""
        import torch

        k, v, sc, rows = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_int64()
        _check(load().refcache_fp8_ptr(self.h, layer, ctypes.byref(k), ctypes.byref(v), ctypes.byref(sc),
                                       ctypes.byref(rows)))
        H, D, n = self.seg.num_heads, self.seg.head_dim, rows.value
        base = self.mem.data_ptr()

        def view(p, nbytes):
            off = p.value - base
            return self.mem[off:off + nbytes]

        return (view(k, n * H * D).view(n, H, D), view(v, n * H * D).view(H, D, n),
                view(sc, (n // 128) * H * 16).view(torch.float32).view(n // 128, H, 4))

    def status(self, stream=None) -> int:
        """Synchronise the stream and return (and clear) this cache's own error
        word as a status code: a bounded wait of one of its launches ran out."""
        return int(load().refcache_cache_status(self.h, _stream(stream)))

    def built(self, layer: int) -> bool:
        r = load().refcache_layer_built(self.h, layer)
        _check(0 if r >= 0 else r)
        return bool(r)

    def launches(self, call: str) -> int:
        """Kernels one build ('build'), step ('step') or in-slot build ('build_in_slot') call launches."""
        r = load().refcache_call_launches(self.h, {"build": 0, "step": 1, "build_in_slot": 2}[call])
        _check(0 if r >= 0 else r)
        return int(r)

    def build(self, layer, q, k, v, o, lse=None, scale=None, stream=None):
        H, D, n = self.seg.num_heads, self.seg.head_dim, self.seg.static_rows
        device = self.mem.get_device()
        ptrs = _thd_ptrs((("q", q), ("k", k), ("v", v), ("o", o)), n, H, D, device)
        scale = default_scale(D) if scale is None else scale
        _check(load().refcache_build(self.h, layer, *ptrs, _ptr(lse, device, "lse"), scale, _stream(stream)))

    def build_in_slot(self, layer, q, k_anchor, v_anchor, o, lse=None, scale=None, stream=None):
        """The prefill of a layer whose cached rows' K/V the caller already
        wrote into the slots (``kv(layer)``); the anchors' K/V are passed apart
        as [sum n_anchor, H, D] (None when there are none, or in the
        alternative anchor reading, whose slots hold them)."""
        H, D, n = self.seg.num_heads, self.seg.head_dim, self.seg.static_rows
        for name, t in (("q", q), ("o", o)):
            _check_thd(name, t, n, H, D)
        n_a = sum(self.seg.n_anchor) if self.mask_mode != "beyond_alt" else 0
        if n_a:
            for name, t in (("k_anchor", k_anchor), ("v_anchor", v_anchor)):
                _check_thd(name, t, n_a, H, D)
        else:
            k_anchor = v_anchor = None
        scale = default_scale(D) if scale is None else scale
        device = self.mem.get_device()
        _check(load().refcache_build_in_slot(self.h, layer, *(_ptr(t, device) for t in (q, k_anchor, v_anchor, o, lse)), scale,
                                             _stream(stream)))

    def step(self, layer, q, k, v, o, lse=None, scale=None, stream=None):
        H, D, n = self.seg.num_heads, self.seg.head_dim, self.seg.live_rows
        device = self.mem.get_device()
        ptrs = _thd_ptrs((("q", q), ("k", k), ("v", v), ("o", o)), n, H, D, device)
        scale = default_scale(D) if scale is None else scale
        _check(load().step_attention(self.h, layer, *ptrs, _ptr(lse, device, "lse"), scale, _stream(stream)))

    def step_backward(self, layer, q, k, v, o, lse, d_o, dq, dk, dv, dk_ref=None, dv_ref=None, accumulate=False, scale=None,
                      stream=None):
        """Gradient of ``step``: from ``d_o``, the gradient of its ``o``, to dq, dk, dv [live rows, H, D] and, unless
        they are None, dk_ref and dv_ref [cached rows, H, D], bf16 or float32 (``accumulate``: added to what these hold; a
        sum over many steps wants float32).  ``lse`` is the fp32 [live rows, H] that the step wrote."""
        H, D, n = self.seg.num_heads, self.seg.head_dim, self.seg.live_rows
        device = self.mem.get_device()
        ptrs, work = _backward_ptrs((q, k, v, o, lse, d_o, dq, dk, dv), n, H, D, device, stream)
        f32, dk_ref, dv_ref = self._ref_ptrs(dk_ref, dv_ref, device)
        scale = default_scale(D) if scale is None else scale
        L = load()
        call = L.step_attention_backward_ref_f32 if f32 else L.step_attention_backward
        _check(call(self.h, layer, *ptrs, dk_ref, dv_ref, 1 if accumulate else 0, work.data_ptr(), scale, _stream(stream)))

    def build_backward(self, layer, q, k, v, o, lse, d_o, dq, dk, dv, dk_ref=None, dv_ref=None, scale=None, stream=None):
        """Gradient of ``build``; dk_ref and dv_ref, the cached rows' gradients from ``step_backward``, are added to
        the cached rows' part of dk and dv unless they are None."""
        H, D, n = self.seg.num_heads, self.seg.head_dim, self.seg.static_rows
        device = self.mem.get_device()
        ptrs, work = _backward_ptrs((q, k, v, o, lse, d_o, dq, dk, dv), n, H, D, device, stream)
        f32, dk_ref, dv_ref = self._ref_ptrs(dk_ref, dv_ref, device)
        scale = default_scale(D) if scale is None else scale
        L = load()
        call = L.refcache_build_backward_ref_f32 if f32 else L.refcache_build_backward
        _check(call(self.h, layer, *ptrs, dk_ref, dv_ref, work.data_ptr(), scale, _stream(stream)))

    def _ref_ptrs(self, dk_ref, dv_ref, device):
        """Whether the cached rows' gradients are float32, and their pointers."""
        if dk_ref is None and dv_ref is None:
            return False, None, None
        n = self.seg.static_rows - (0 if self.mask_mode == "beyond_alt" else sum(self.seg.n_anchor))  # cached rows
        H, D = self.seg.num_heads, self.seg.head_dim
        if dk_ref is None or dk_ref.dtype is not _float32:
            k, v = _thd_ptrs((("dk_ref", dk_ref), ("dv_ref", dv_ref)), n, H, D, device)
            return False, k, v
        shape = (n, H, D)
        for name, t in (("dk_ref", dk_ref), ("dv_ref", dv_ref)):
            if t is None or t.dtype is not _float32 or t.shape != shape:
                got = None if t is None else f"{t.dtype} {tuple(t.shape)}"
                raise ValueError(f"{name}: expected float32 {list(shape)} beside the other, got {got}")
        return True, _ptr(dk_ref, device, "dk_ref"), _ptr(dv_ref, device, "dv_ref")


def full_attention(cu_seqlens, q, k, v, o, lse=None, scale=None, stream=None):
    rows, H, D = q.shape
    cu = list(cu_seqlens)
    device = _device()
    ptrs = _thd_ptrs((("q", q), ("k", k), ("v", v), ("o", o)), cu[-1], H, D, device)
    scale = default_scale(D) if scale is None else scale
    _check(load().full_attention(len(cu) - 1, H, D, _arr(cu), *ptrs, _ptr(lse, device, "lse"), scale, _stream(stream)))


def full_attention_noalloc(cu_seqlens, q, k, v, o, lse=None, scale=None, stream=None):
    """full_attention whose work list sits in the library's static device
    memory: the call allocates no device memory (see include/refcache.h)."""
    rows, H, D = q.shape
    cu = list(cu_seqlens)
    device = _device()
    ptrs = _thd_ptrs((("q", q), ("k", k), ("v", v), ("o", o)), cu[-1], H, D, device)
    scale = default_scale(D) if scale is None else scale
    _check(load().full_attention_noalloc(len(cu) - 1, H, D, _arr(cu), *ptrs, _ptr(lse, device, "lse"), scale, _stream(stream)))


# torch, bfloat16, float32 and int32, once torch is in use (an import statement in a
# function costs as much as checking a tensor)
_torch = _bfloat16 = _float32 = _int32 = None


def _use_torch():
    global _torch, _bfloat16, _float32, _int32
    import torch

    _torch, _bfloat16, _float32, _int32 = torch, torch.bfloat16, torch.float32, torch.int32


def _empty(shape, dtype, device, stream):
    """Memory for a call on ``stream`` from torch's allocator, of that stream's own blocks: what was freed on the current
    stream may still be in use there, and what this call leaves goes on only to work behind it."""
    if stream is None:
        return _torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, _torch.cuda.Stream):
        stream = _torch.cuda.ExternalStream(_stream(stream), device=device)
    with _torch.cuda.stream(stream):
        return _torch.empty(shape, dtype=dtype, device=device)


def _work(nbytes, like, stream):
    """A call's workspace."""
    return _empty(max(16, nbytes), _torch.uint8, like.device, stream)


_BACKWARD = ("q", "k", "v", "o", "lse", "d_o", "dq", "dk", "dv")


def _backward_ptrs(tensors, rows, H, D, device, stream):
    """The device pointers of a gradient call's tensors, in their order, and its workspace."""
    if _torch is None:
        _use_torch()
    shape, lse = (rows, H, D), tensors[4]
    if lse is None:
        raise ValueError("lse is required")
    if lse.dtype is not _float32 or lse.shape != (rows, H):
        raise ValueError(f"lse: expected float32 [{rows}, {H}], got {lse.dtype} {tuple(lse.shape)}")
    ptrs = []
    for t in tensors:
        if t is not lse and (t is None or t.dtype is not _bfloat16 or t.shape != shape):
            _check_thd(_BACKWARD[len(ptrs)], t, rows, H, D)
        if t.get_device() != device or not t.is_contiguous():
            _ptr(t, device, _BACKWARD[len(ptrs)])
        ptrs.append(t.data_ptr())
    return ptrs, _work(load().refcache_backward_bytes(rows, H), lse, stream)


def full_attention_backward(cu_seqlens, q, k, v, o, lse, d_o, dq, dk, dv, scale=None, stream=None):
    """Gradient of ``full_attention`` (of either allocation variant)."""
    _, H, D = q.shape
    cu = list(cu_seqlens)
    ptrs, work = _backward_ptrs((q, k, v, o, lse, d_o, dq, dk, dv), cu[-1], H, D, _device(), stream)
    scale = default_scale(D) if scale is None else scale
    _check(load().full_attention_backward(len(cu) - 1, H, D, _arr(cu), *ptrs, work.data_ptr(), scale, _stream(stream)))


class Rope:
    """Rotary positions with several axes (refcache_rope_t): ``axes`` are the dims of a head that each axis turns."""

    def __init__(self, head_dim, axes, theta=10000.0, pairs="interleaved"):
        if pairs not in ROPE_PAIRS:
            raise ValueError(f"pairs: expected one of {sorted(ROPE_PAIRS)}, got {pairs!r}")
        self.head_dim, self.axes, self.theta, self.pairs = int(head_dim), tuple(int(a) for a in axes), float(theta), pairs
        self.c = _Rope()
        _check(load().refcache_rope_init(ctypes.byref(self.c), self.head_dim, len(self.axes), _arr(self.axes), self.theta,
                                         ROPE_PAIRS[pairs]))
        self._ref = ctypes.byref(self.c)


_NOTHING = 16  # the address of a tensor without elements, which torch gives as NULL; nothing is read or written there


def _rows_apart(names, tensors, shape, device):
    """For each tensor its pointer and the elements between its rows: [rows, H, D] bf16 whose rows are contiguous."""
    n, H, D = shape
    out = []
    for name, t in zip(names, tensors):
        if t is None:
            out += (None, H * D)
            continue
        if t.dtype is not _bfloat16 or t.shape != shape:
            raise ValueError(f"{name}: expected bf16 {list(shape)}, got {t.dtype} {tuple(t.shape)}")
        if t.get_device() != device:
            raise _elsewhere(t, device, name)
        s = t.stride()
        if s[2] != 1 or (s[1] != D and H > 1):
            raise ValueError(f"{name}: the heads of a row must be contiguous, got strides {s}")
        out += (t.data_ptr() or _NOTHING, s[0] if n > 1 else H * D)
    return out


def _rows_packed(names, tensors, shape, device):
    out = []
    for name, t in zip(names, tensors):
        if t is None:
            out.append(None)
            continue
        if t.dtype is not _bfloat16 or t.shape != shape or t.get_device() != device or not t.is_contiguous():
            _check_thd(name, t, *shape)
            _ptr(t, device, name)
        out.append(t.data_ptr() or _NOTHING)
    return out


def _param(name, t, n, f32, device):
    """The pointer of a contiguous [n] parameter in bf16 or fp32, and whether it is fp32 (``f32``: that of one before)."""
    if t is None:
        return None, f32
    is32 = t.dtype is _float32
    if not (is32 or t.dtype is _bfloat16) or t.shape != (n,):
        raise ValueError(f"{name}: expected bf16 or float32 [{n}], got {t.dtype} {tuple(t.shape)}")
    if f32 is not None and f32 != is32:
        raise ValueError(f"{name}: the parameters of one call have one type")
    return _ptr(t, device, name), is32


def _rope_rows(rope, positions, shape, out_rows, wq, wk, rows, eps, device):
    n, H, _ = shape
    if positions.dtype is not _int32 or positions.shape != (n, len(rope.axes)):
        raise ValueError(f"positions: expected int32 [{n}, {len(rope.axes)}], got {positions.dtype} {tuple(positions.shape)}")
    if rows is not None and (rows.dtype is not _int32 or rows.shape != (n,)):
        raise ValueError(f"rows: expected int32 [{n}], got {rows.dtype} {tuple(rows.shape)}")
    pq, f32 = _param("weight_q", wq, rope.head_dim, None, device)
    pk, f32 = _param("weight_k", wk, rope.head_dim, f32, device)
    return _RopeRows(n, out_rows, H, 1 if f32 else 0, _ptr(positions, device, "positions"), _ptr(rows, device, "rows"), pq, pk, eps)


def _shape_of(what, a, b, c):
    """The [rows, H, D] of the first of three tensors that is there."""
    t = a if a is not None else b if b is not None else c
    if t is None:
        raise ValueError(f"{what}: none of the three tensors is there")
    if t.dim() != 3:
        raise ValueError(f"{what}: expected [rows, heads, dim], got {tuple(t.shape)}")
    return t.shape


def qkv_rope(rope, positions, q, k, v, q_out, k_out, v_out, weight_q=None, weight_k=None, rows=None, eps=1e-6, stream=None):
    """From a projection's q, k and v ([rows, H, D] bf16, rows may lie apart, as those of a fused projection do) to the
    attention's ([out rows, H, D], packed): RMS norm of each head of q and k (with a weight), rotary positions, row i
    moved to row ``rows[i]``.  q, k or v may be None together with its output."""
    if _torch is None:
        _use_torch()
    n, H, _ = _shape_of("qkv_rope", q, k, v)
    out = _shape_of("qkv_rope's outputs", q_out, k_out, v_out)[0]
    D, device = rope.head_dim, _device()
    r = _rope_rows(rope, positions, (n, H, D), out, weight_q, weight_k, rows, eps, device)
    src = _rows_apart(("q", "k", "v"), (q, k, v), (n, H, D), device)
    dst = _rows_packed(("q_out", "k_out", "v_out"), (q_out, k_out, v_out), (out, H, D), device)
    _check(load().refcache_qkv_rope(rope._ref, ctypes.byref(r), *src, *dst, _stream(stream)))


def qkv_rope_backward(rope, positions, q, k, dq_out, dk_out, dv_out, dq, dk, dv, weight_q=None, weight_k=None, dweight_q=None,
                      dweight_k=None, rows=None, eps=1e-6, stream=None):
    """Gradient of ``qkv_rope``: from those of its outputs to dq, dk and dv (rows may lie apart) and the weights' (fp32
    [D]).  q and k are its inputs, needed where they were normalised."""
    if _torch is None:
        _use_torch()
    n, H, _ = _shape_of("qkv_rope_backward", dq, dk, dv)
    out = _shape_of("qkv_rope_backward's inputs", dq_out, dk_out, dv_out)[0]
    D, device = rope.head_dim, _device()
    r = _rope_rows(rope, positions, (n, H, D), out, weight_q, weight_k, rows, eps, device)
    src = _rows_apart(("q", "k"), (q, k), (n, H, D), device)
    grad = _rows_packed(("dq_out", "dk_out", "dv_out"), (dq_out, dk_out, dv_out), (out, H, D), device)
    dst = _rows_apart(("dq", "dk", "dv"), (dq, dk, dv), (n, H, D), device)
    L = load()
    dw, work = [], None
    for name, t in (("dweight_q", dweight_q), ("dweight_k", dweight_k)):
        if t is not None and (t.dtype is not _float32 or t.shape != (D,)):
            raise ValueError(f"{name}: expected float32 [{D}], got {t.dtype} {tuple(t.shape)}")
        dw.append(_ptr(t, device, name))
    if weight_q is not None or weight_k is not None:
        work = _work(L.refcache_qkv_rope_backward_bytes(rope._ref), positions, stream)
    _check(L.refcache_qkv_rope_backward(rope._ref, ctypes.byref(r), *src, *grad, *dst, *dw, None if work is None else work.data_ptr(),
                                        _stream(stream)))


def _norm_params(cu_rows, width, gate, scale, shift, weight, post_weight, norm, post_norm, eps, device):
    cu = list(cu_rows)
    batch = len(cu) - 1
    shape, f32, ptrs, lds = (batch, width), None, [], []
    for name, t in (("gate", gate), ("scale", scale), ("shift", shift)):
        if t is None:
            ptrs.append(None)
            lds.append(0)
            continue
        is32 = t.dtype is _float32
        if not (is32 or t.dtype is _bfloat16) or t.shape != shape:
            raise ValueError(f"{name}: expected bf16 or float32 {list(shape)}, got {t.dtype} {tuple(t.shape)}")
        if f32 is not None and f32 != is32:
            raise ValueError(f"{name}: the parameters of one call have one type")
        if t.get_device() != device:
            raise _elsewhere(t, device, name)
        s = t.stride()
        if s[1] != 1:
            raise ValueError(f"{name}: its rows must be contiguous")
        f32 = is32
        ptrs.append(t.data_ptr())
        lds.append(s[0] if batch > 1 else width)
    w, f32 = _param("weight", weight, width, f32, device)
    pw, f32 = _param("post_weight", post_weight, width, f32, device)
    return _GatedNorm(batch, width, _arr(cu), NORMS[norm], NORMS[post_norm], 1 if f32 else 0, eps, *ptrs, *lds, w, pw)


def _row_ptrs(names, tensors, shape, device):
    out = []
    for name, t in zip(names, tensors):
        if t is None:
            out.append(None)
            continue
        if t.dtype is not _bfloat16 or t.shape != shape:
            raise ValueError(f"{name}: expected bf16 {list(shape)}, got {t.dtype} {tuple(t.shape)}")
        out.append(_ptr(t, device, name))
    return out


def gated_norm(cu_rows, x, y=None, branch=None, x_out=None, gate=None, scale=None, shift=None, weight=None, post_weight=None,
               norm="layer", post_norm=None, eps=1e-6, stream=None):
    """x_out = x + gate * h with h = branch, or its ``post_norm`` times post_weight; y = norm(x_out) * weight *
    (1 + scale) + shift.  x, branch, x_out (may be x) and y: [rows, width] bf16, packed; gate, scale and shift: a row for
    each request of ``cu_rows``, rows may lie apart or be one expanded row; norms "layer", "rms" or None."""
    if _torch is None:
        _use_torch()
    width, device = x.shape[1], _device()
    c = _norm_params(cu_rows, width, gate, scale, shift, weight, post_weight, norm, post_norm, eps, device)
    ptrs = _row_ptrs(("x", "branch", "x_out", "y"), (x, branch, x_out, y), (cu_rows[-1], width), device)
    _check(load().refcache_gated_norm(ctypes.byref(c), *ptrs, _stream(stream)))


def gated_norm_backward(cu_rows, x_out, dy, dx, branch=None, dx_out=None, d_branch=None, gate=None, scale=None, weight=None,
                        post_weight=None, d_gate=None, d_scale=None, d_shift=None, d_weight=None, d_post_weight=None,
                        norm="layer", post_norm=None, eps=1e-6, stream=None):
    """Gradient of ``gated_norm``: from dy and dx_out, the gradients of its outputs (either may be None), to dx, d_branch,
    the modulation's (fp32 [requests, width]) and the weights' (fp32 [width]), each unless it is None.  ``x_out`` is the
    call's output (its x where there was no branch)."""
    if _torch is None:
        _use_torch()
    like = dy if dy is not None else dx_out
    if like is None:
        raise ValueError("gated_norm_backward needs dy or dx_out")
    width, device = like.shape[1], _device()
    c = _norm_params(cu_rows, width, gate, scale, None, weight, post_weight, norm, post_norm, eps, device)
    ptrs = _row_ptrs(("x_out", "branch", "dy", "dx_out", "dx", "d_branch"), (x_out, branch, dy, dx_out, dx, d_branch), (cu_rows[-1], width), device)
    sums = []
    for name, t in (("d_gate", d_gate), ("d_scale", d_scale), ("d_shift", d_shift), ("d_weight", d_weight), ("d_post_weight", d_post_weight)):
        shape = (c.batch, width) if len(sums) < 3 else (width,)
        if t is not None and (t.dtype is not _float32 or t.shape != shape):
            raise ValueError(f"{name}: expected float32 {list(shape)}, got {t.dtype} {tuple(t.shape)}")
        sums.append(_ptr(t, device, name))
    L, ref = load(), ctypes.byref(c)
    work = _work(L.refcache_gated_norm_backward_bytes(ref), like, stream)
    _check(L.refcache_gated_norm_backward(ref, *ptrs, *sums, work.data_ptr(), _stream(stream)))


def clip_gradients(grads, max_norm, out=None, norm=None, stream=None):
    """Scales gradients (bf16 or float32 tensors of any shapes) so that their global norm is at most ``max_norm``, in
    place or into the tensors ``out``; returns the norm before (float32, on the GPU; ``norm`` if given).  max_norm
    may be infinite: the norm alone, the gradients as they are."""
    if _torch is None:
        _use_torch()
    grads = list(grads)
    n = len(grads)
    outs = None if out is None else list(out)
    if outs is not None and len(outs) != n:
        raise ValueError(f"{n} gradients and {len(outs)} outputs")
    counts = [g.numel() for g in grads]
    if outs is not None and [o.numel() for o in outs] != counts:
        i, o = next((i, o) for i, (m, o) in enumerate(zip(counts, outs)) if o.numel() != m)
        raise ValueError(f"gradient {i}: {counts[i]} elements and an output of {o.numel()}")
    device = _device()
    for tensors in (grads,) if outs is None else (grads, outs):
        for i, t in enumerate(tensors):
            if t.get_device() != device or not t.is_contiguous():
                _ptr(t, device, f"gradient {i}")
    kind = {_bfloat16: 0, _float32: 1}
    try:
        types = [kind[g.dtype] for g in grads]
        types = [3 * t for t in types] if outs is None else [t + 2 * kind[o.dtype] for t, o in zip(types, outs)]
    except KeyError as e:
        raise ValueError(f"gradients: expected bf16 or float32, got {e.args[0]}") from None
    if norm is None:
        norm = _empty((), _float32, grads[0].device if grads else _torch.device("cuda", device), stream)
    elif norm.dtype is not _float32 or norm.numel() != 1:
        raise ValueError(f"norm: expected one float32, got {norm.dtype} {tuple(norm.shape)}")
    norm_ptr = _ptr(norm, device, "norm")
    L = load()
    work = _work(L.refcache_clip_gradients_bytes(n), norm, stream)
    # (arrays of the array module: ctypes' took half of the time that a tensor costs)
    lists = [array("Q", [g.data_ptr() for g in grads]), None if outs is None else array("Q", [o.data_ptr() for o in outs]),
             array("q", counts), array("i", types)]
    _check(L.refcache_clip_gradients(n, *[None if a is None else a.buffer_info()[0] for a in lists], max_norm, norm_ptr,
                                     work.data_ptr(), _stream(stream)))
    return norm
