"""Refusals of the gradients' and block operators' entry points, which come before a device is touched."""
import ctypes
import math

import pytest

from paper_2608_21229_gb300 import build as cbuild
from paper_2608_21229_gb300 import refcache as rcb


@pytest.fixture(scope="module")
def lib():
    cbuild.build()
    return rcb.load()


def test_rope_tables(lib):
    r = rcb.Rope(128, (16, 56, 56), theta=10000.0)
    assert list(r.c.axis) == [0] * 8 + [1] * 28 + [2] * 28
    for j, (i, k, a) in enumerate([(0, k, 16) for k in range(8)] + [(1, k, 56) for k in range(28)]):
        turns = 10000.0 ** (-2 * k / a) / (2 * math.pi)
        assert abs(r.c.turn_hi[j] + r.c.turn_lo[j] - turns) <= 2.0 ** -46 * turns
    part = rcb.Rope(64, (0, 20))
    assert list(part.c.turn_hi)[10:] == [0.0] * 54


@pytest.mark.parametrize("kw", [dict(head_dim=96, axes=(96,)), dict(head_dim=64, axes=(64, 2)), dict(head_dim=64, axes=(3,)),
                                dict(head_dim=64, axes=(-2, 4)), dict(head_dim=64, axes=()), dict(head_dim=64, axes=(2,) * 5),
                                dict(head_dim=64, axes=(64,), theta=0.0), dict(head_dim=64, axes=(64,), theta=math.inf)])
def test_rope_refusals(lib, kw):
    with pytest.raises(rcb.RefCacheError):
        rcb.Rope(**kw)


def test_pairs_by_name(lib):
    with pytest.raises(ValueError, match="pairs"):
        rcb.Rope(64, (64,), pairs="both")


P = 0x1000  # an aligned address that is never read


def rope_rows(**kw):
    d = dict(rows=4, out_rows=4, num_heads=2, weight_f32=0, positions=P, row_map=None, weight_q=None, weight_k=None, eps=1e-6)
    d.update(kw)
    return rcb._RopeRows(**d)


@pytest.mark.parametrize("rows, ld, ptr", [
    (dict(rows=-1), 128, P), (dict(num_heads=0), 128, P), (dict(out_rows=3), 128, P), (dict(positions=None), 128, P),
    (dict(eps=-1.0), 128, P), (dict(eps=math.nan), 128, P), (dict(weight_q=P + 2), 128, P), ({}, 120, P), ({}, 132, P), ({}, 128, P + 2),
    (dict(num_heads=1 << 20), 1 << 27, P), (dict(row_map=P + 1), 128, P),
])
def test_qkv_rope_refusals(lib, rows, ld, ptr):
    rope, r = rcb.Rope(64, (64,)), rope_rows(**rows)
    args = (ctypes.byref(rope.c), ctypes.byref(r), ptr, ld, None, 0, None, 0, P, None, None, None)
    assert lib.refcache_qkv_rope(*args) == rcb.ERR_INVALID_ARG and rcb.last_error()
    empty = rcb._Rope()
    assert lib.refcache_qkv_rope(ctypes.byref(empty), *args[1:]) in (rcb.ERR_INVALID_ARG, rcb.ERR_UNSUPPORTED)


def test_qkv_rope_backward_refusals(lib):
    rope, r, w = rcb.Rope(64, (64,)), rope_rows(), rope_rows(weight_q=P)
    f = lib.refcache_qkv_rope_backward
    go = lambda rows, **kw: f(ctypes.byref(rope.c), ctypes.byref(rows), *{  # noqa: E731
        **dict(q=P, ldq=128, k=None, ldk=0, gq=P, gk=None, gv=None, dq=P, lddq=128, dk=None, lddk=0, dv=None, lddv=0, wq=None, wk=None,
               work=P, s=None), **kw}.values())
    for rows, kw in ((r, dict(dq=None)), (r, dict(gv=P)), (r, dict(wq=P)), (r, dict(lddq=64)), (w, dict(q=None)), (w, dict(ldq=100)),
                     (w, dict(work=None)), (w, dict(wk=P)), (w, dict(work=P + 4))):
        assert go(rows, **kw) == rcb.ERR_INVALID_ARG, kw


def norm_params(cu=(0, 2, 4), **kw):
    arr = (ctypes.c_int32 * len(cu))(*cu)
    d = dict(batch=len(cu) - 1, width=64, cu_rows=arr, norm=1, post_norm=0, mod_f32=0, eps=1e-6)
    d.update(kw)
    c = rcb._GatedNorm(**d)
    c._keep = arr
    return c


@pytest.mark.parametrize("kw", [dict(width=12), dict(width=0), dict(width=8200), dict(batch=0), dict(cu=(1, 2)), dict(cu=(0, 3, 2)),
                                dict(norm=3), dict(post_norm=-1), dict(eps=-1.0), dict(gate=P, ld_gate=56), dict(gate=P, ld_gate=68),
                                dict(scale=P + 2, ld_scale=64), dict(weight=P + 8), dict(post_weight=P)])
def test_gated_norm_refusals(lib, kw):
    c = norm_params(**kw)
    assert lib.refcache_gated_norm(ctypes.byref(c), P, P, P, P, None) in (rcb.ERR_INVALID_ARG, rcb.ERR_UNSUPPORTED)
    assert lib.refcache_gated_norm_backward_bytes(ctypes.byref(c)) == 0


def test_gated_norm_tensor_refusals(lib):
    c, w = norm_params(), norm_params(weight=P)
    f = lib.refcache_gated_norm
    assert f(ctypes.byref(c), None, P, P, P, None) == rcb.ERR_INVALID_ARG
    assert f(ctypes.byref(c), P + 8, P, P, P, None) == rcb.ERR_INVALID_ARG
    assert f(ctypes.byref(c), P, None, P, P, None) == rcb.ERR_INVALID_ARG
    b = lib.refcache_gated_norm_backward
    names = ("x_out", "branch", "dy", "dx_out", "dx", "d_branch", "d_gate", "d_scale", "d_shift", "d_weight", "d_post_weight", "work")
    go = lambda p, **kw: b(ctypes.byref(p), *[kw.get(n, P) for n in names], None)  # noqa: E731
    base = dict(d_weight=None, d_post_weight=None)
    for p, kw in ((c, dict(x_out=None)), (c, dict(branch=None)), (c, dict(dy=None, dx_out=None)), (c, dict(work=None)), (c, dict(d_weight=P)),
                  (w, dict(d_post_weight=P)), (c, dict(dx=P + 2))):
        assert go(p, **{**base, **kw}) == rcb.ERR_INVALID_ARG, kw


def test_float_results_are_aligned(lib):
    """A float32 result at an odd address is refused, not written."""
    rope, w = rcb.Rope(64, (64,)), rope_rows(weight_q=P)
    assert lib.refcache_qkv_rope_backward(ctypes.byref(rope.c), ctypes.byref(w), P, 128, None, 0, P, None, None, P, 128, None, 0, None, 0,
                                          P + 2, None, P, None) == rcb.ERR_INVALID_ARG
    c = norm_params(weight=P, post_weight=P, post_norm=2)
    for i in range(5):
        sums = [P + 1 if j == i else P for j in range(5)]
        assert lib.refcache_gated_norm_backward(ctypes.byref(c), P, P, P, P, P, P, *sums, P, None) == rcb.ERR_INVALID_ARG, i
    ok = ((ctypes.c_void_p * 1)(P), None, (ctypes.c_int64 * 1)(4), (ctypes.c_int32 * 1)(0))
    assert lib.refcache_clip_gradients(1, *ok, 1.0, P + 2, P, None) == rcb.ERR_INVALID_ARG


def test_clip_refusals(lib):
    vp, i64, i32 = ctypes.c_void_p * 1, ctypes.c_int64 * 1, ctypes.c_int32 * 1
    f = lib.refcache_clip_gradients
    ok = (vp(P), None, i64(4), i32(0))
    assert f(-1, *ok, 1.0, None, P, None) == rcb.ERR_INVALID_ARG
    assert f(1, None, None, i64(4), i32(0), 1.0, None, P, None) == rcb.ERR_INVALID_ARG
    assert f(1, *ok, -1.0, None, P, None) == rcb.ERR_INVALID_ARG
    assert f(1, *ok, math.nan, None, P, None) == rcb.ERR_INVALID_ARG
    assert f(1, *ok, 1.0, None, None, None) == rcb.ERR_INVALID_ARG
    for bad in ((vp(P), None, i64(-1), i32(0)), (vp(P), None, i64(4), i32(4)), (vp(P + 1), None, i64(4), i32(0)), (vp(None), None, i64(4), i32(0)),
                (vp(P), None, i64(4), i32(2)), (vp(P), vp(P + 2), i64(4), i32(2))):
        assert f(1, *bad, 1.0, None, P, None) == rcb.ERR_INVALID_ARG, bad


def test_attention_gradient_refusals(lib):
    cu = (ctypes.c_int32 * 2)(0, 16)
    f = lib.full_attention_backward
    t = [P] * 10  # q, k, v, o, lse, d_o, dq, dk, dv, work
    assert f(1, 4, 96, cu, *t, 0.1, None) == rcb.ERR_UNSUPPORTED
    assert f(0, 4, 64, cu, *t, 0.1, None) == rcb.ERR_INVALID_ARG
    assert f(1, 4, 64, cu, *t, -0.1, None) == rcb.ERR_INVALID_ARG
    for i in range(10):
        assert f(1, 4, 64, cu, *t[:i], None, *t[i + 1:], 0.1, None) == rcb.ERR_INVALID_ARG, i
        assert f(1, 4, 64, cu, *t[:i], P + 2, *t[i + 1:], 0.1, None) == rcb.ERR_INVALID_ARG, i
    assert lib.step_attention_backward(None, 0, *[P] * 11, 0, P, 0.1, None) == rcb.ERR_INVALID_ARG
    assert lib.refcache_build_backward(None, 0, *[P] * 12, 0.1, None) == rcb.ERR_INVALID_ARG
    assert lib.refcache_backward_bytes(100, 24) >= 100 * 24 * 8 and lib.refcache_backward_bytes(-1, 2) == 0
