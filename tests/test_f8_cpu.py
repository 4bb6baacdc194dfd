"""Refusals of the 8-bit linear layers' entry points, which come before a device is touched."""
import ctypes

import pytest

from paper_2608_21229_gb300 import build as cbuild
from paper_2608_21229_gb300 import refcache as rcb

P = 0x1000  # an aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    cbuild.build()
    return rcb.load()


def rows(n=4, width=64, codes=P, scales=P, tiles=P):
    return ctypes.byref(rcb._F8Rows(n, width, codes, scales, tiles))


def weight(out=32, inn=64, codes=P, scales=P, tiles=P, codes_t=P, scales_t=P, tiles_t=P):
    return ctypes.byref(rcb._F8Weight(out, inn, codes, scales, tiles, codes_t, scales_t, tiles_t))


BAD_ROWS = [dict(n=-1), dict(n=(1 << 31) - 1), dict(width=0), dict(width=24), dict(width=(1 << 20) + 16), dict(codes=None), dict(scales=None),
            dict(codes=P + 8), dict(scales=P + 4), dict(tiles=None), dict(tiles=P + 8)]
BAD_WEIGHT = [dict(out=0), dict(out=40), dict(inn=-16), dict(inn=(1 << 20) + 16)]
INVALID = rcb.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", BAD_ROWS, ids=str)
def test_rows_refusals(lib, kw):
    bad = rows(**kw)
    assert lib.refcache_f8_quantize(P, 1 << 21, bad, None) == INVALID and rcb.last_error()
    w = kw.get("width", 64)
    n = kw.get("n", 4)
    assert lib.refcache_f8_linear(bad, weight(inn=w if w > 0 and w % 16 == 0 else 64), 0, None, 0, P, 64, None) == INVALID
    assert lib.refcache_f8_linear_gelu(bad, weight(), None, 0, 0, rows(n, 32), None, None) == INVALID
    assert lib.refcache_f8_linear_gelu(rows(), weight(), None, 0, 0, bad, None, None) == INVALID
    assert lib.refcache_f8_linear_gelu(rows(), weight(), None, 0, 0, rows(width=32), bad, None) == INVALID
    assert lib.refcache_f8_linear_gelu_backward(bad, weight(), 0, rows(), P, 64, None, None) == INVALID
    assert lib.refcache_f8_linear_gelu_backward(rows(width=32), weight(), 0, bad, P, 64, None, None) == INVALID
    assert lib.refcache_f8_linear_gelu_backward(rows(width=32), weight(), 0, rows(), P, 64, bad, None) == INVALID
    assert lib.refcache_f8_weight_grad(P, 1 << 10, bad, 64, None, P, 1, None, P, None) == INVALID


@pytest.mark.parametrize("kw", BAD_WEIGHT, ids=str)
def test_weight_refusals(lib, kw):
    bad = weight(**kw)
    assert lib.refcache_f8_quantize_weight(P, 0, bad, None) == INVALID
    assert lib.refcache_f8_linear(rows(), bad, 0, None, 0, P, 64, None) == INVALID
    assert lib.refcache_f8_linear(rows(width=32), bad, 1, None, 0, P, 64, None) == INVALID
    assert lib.refcache_f8_linear_gelu(rows(), bad, None, 0, 0, rows(width=32), None, None) == INVALID
    assert lib.refcache_f8_linear_gelu_backward(rows(width=32), bad, 0, rows(), P, 64, None, None) == INVALID


def test_missing_orientation_refusals(lib):
    for kw in (dict(codes=None), dict(scales=None), dict(tiles=None), dict(codes=P + 8), dict(scales=P + 8), dict(tiles=P + 8)):
        assert lib.refcache_f8_linear(rows(), weight(**kw), 0, None, 0, P, 64, None) == INVALID
        assert lib.refcache_f8_linear_gelu(rows(), weight(**kw), None, 0, 0, rows(width=32), None, None) == INVALID
        assert lib.refcache_f8_quantize_weight(P, 0, weight(**kw), None) == INVALID
    for kw in (dict(codes_t=None), dict(scales_t=None), dict(tiles_t=None), dict(codes_t=P + 8), dict(scales_t=P + 8), dict(tiles_t=P + 8)):
        assert lib.refcache_f8_linear(rows(width=32), weight(**kw), 1, None, 0, P, 64, None) == INVALID
        assert lib.refcache_f8_linear_gelu_backward(rows(width=32), weight(**kw), 0, rows(), P, 64, None, None) == INVALID
        assert lib.refcache_f8_quantize_weight(P, 0, weight(**kw), None) == INVALID


def test_tensor_refusals(lib):
    q, lin, gelu = lib.refcache_f8_quantize, lib.refcache_f8_linear, lib.refcache_f8_linear_gelu
    back, wg = lib.refcache_f8_linear_gelu_backward, lib.refcache_f8_weight_grad
    for x, ld in ((None, 64), (P + 2, 64), (P, 56), (P, 68), (P, 1 << 33)):
        assert q(x, ld, rows(), None) == INVALID
    for y, ld in ((None, 32), (P + 2, 32), (P, 24), (P, 36), (P, 0)):
        assert lin(rows(), weight(), 0, None, 0, y, ld, None) == INVALID
    assert lin(None, weight(), 0, None, 0, P, 32, None) == INVALID and lin(rows(), None, 0, None, 0, P, 32, None) == INVALID
    assert lin(rows(width=48), weight(), 0, None, 0, P, 32, None) == INVALID  # another width than the weight's
    assert lin(rows(), weight(), 1, None, 0, P, 64, None) == INVALID
    assert lin(rows(), weight(), 0, P + 1, 0, P, 32, None) == INVALID and lin(rows(), weight(), 0, P + 2, 1, P, 32, None) == INVALID
    assert gelu(rows(), weight(), None, 0, 2, rows(width=32), None, None) == INVALID  # unknown form
    assert gelu(rows(), weight(), None, 0, 0, rows(5, 32), None, None) == INVALID
    assert gelu(rows(), weight(), None, 0, 0, rows(width=32), rows(3, 32), None) == INVALID
    assert gelu(rows(), weight(), None, 0, 0, None, rows(width=32), None) == INVALID
    assert back(rows(width=32), weight(), -1, rows(), P, 64, None, None) == INVALID
    assert back(rows(width=32), weight(), 0, rows(), None, 64, None, None) == INVALID  # nothing to write
    assert back(rows(width=32), weight(), 0, rows(), P + 8, 64, None, None) == INVALID
    assert back(rows(width=32), weight(), 0, rows(), P, 56, None, None) == INVALID
    assert back(rows(width=32), weight(), 0, rows(5), P, 64, None, None) == INVALID
    assert back(rows(width=32), weight(), 0, None, P, 64, None, None) == INVALID
    ok = dict(dy=P, ld=32, x=rows(), n=32, add=None, dw=P, f32=1, db=None, work=P, s=None)
    for kw in (dict(dy=None), dict(dy=P + 2), dict(ld=24), dict(ld=33), dict(x=None), dict(n=0), dict(n=24), dict(add=P + 4), dict(dw=None),
               dict(dw=P + 4), dict(db=P + 2)):
        assert wg(*{**ok, **kw}.values()) == INVALID, kw
    assert q(P, 64, None, None) == INVALID and lib.refcache_f8_quantize_weight(None, 0, weight(), None) == INVALID
    assert lib.refcache_f8_quantize_weight(P + 8, 1, weight(), None) == INVALID


def at(i):
    """Addresses that are never read, 16 MB apart."""
    return 0x1000000 * i


def test_overlaps_are_refused(lib):
    """An output on an input or on another output, wholly or in part, before a device is touched."""
    q, qw, lin, gelu = lib.refcache_f8_quantize, lib.refcache_f8_quantize_weight, lib.refcache_f8_linear, lib.refcache_f8_linear_gelu
    back, wg = lib.refcache_f8_linear_gelu_backward, lib.refcache_f8_weight_grad

    def form(i, n=4, width=64, **kw):
        return rows(n, width, **{**dict(codes=at(i), scales=at(i + 1), tiles=at(i + 2)), **kw})

    def w(i, **kw):
        return weight(64, 64, **{**dict(codes=at(i), scales=at(i + 1), tiles=at(i + 2), codes_t=at(i + 3), scales_t=at(i + 4), tiles_t=at(i + 5)), **kw})

    def refused(status):
        assert status == INVALID and "overlap" in rcb.last_error()

    refused(q(at(1), 64, form(1), None))
    refused(q(at(1) + 240, 64, form(2, codes=at(1)), None))  # codes of 256 bytes
    refused(q(at(1), 64, form(2, tiles=at(1) + 256), None))
    refused(q(at(9), 64, form(2, scales=at(2) + 240), None))  # scales in the codes
    refused(qw(at(1), 1, w(1), None))
    refused(qw(at(9), 0, w(1, codes_t=at(1) + 4080), None))
    refused(lin(form(1), w(10), 0, None, 0, at(1), 64, None))
    refused(lin(form(1), w(10), 0, None, 0, at(12), 64, None))
    refused(lin(form(1), w(10), 1, None, 0, at(13), 64, None))
    refused(lin(form(1), w(10), 0, at(20), 0, at(20) + 112, 64, None))
    refused(gelu(form(1), w(10), None, 0, 0, form(1), None, None))
    refused(gelu(form(1), w(10), None, 0, 0, form(4), form(4), None))
    refused(gelu(form(1), w(10), None, 0, 0, form(4), form(6), None))  # a's tiles are u's codes
    refused(back(form(1), w(10), 0, form(4), at(20), 64, form(4), None))
    refused(back(form(1), w(10), 0, form(4), at(20), 64, form(1), None))
    refused(back(form(1), w(10), 0, form(4), at(4), 64, None, None))
    refused(back(form(1), w(10), 0, form(4), at(20), 64, form(20), None))
    args = dict(dy=at(1), ld=64, x=form(2), n=64, add=None, dw=at(5), f32=1, db=at(6), work=at(7), s=None)
    for kw in (dict(dw=at(1)), dict(dw=at(2)), dict(db=at(1) + 508), dict(db=at(5) + 16128), dict(work=at(2)), dict(work=at(5)), dict(add=at(5) + 16),
               dict(add=at(7))):
        refused(wg(*{**args, **kw}.values()))


def test_calls_without_rows_need_no_tensors(lib):
    """Nothing to do: accepted before a device is asked for."""
    empty = lambda w: rows(0, w, None, None, None)  # noqa: E731
    assert lib.refcache_f8_quantize(None, 64, empty(64), None) == rcb.OK
    assert lib.refcache_f8_linear(empty(64), weight(), 0, None, 0, None, 32, None) == rcb.OK
    assert lib.refcache_f8_linear_gelu(empty(64), weight(), None, 0, 0, empty(32), empty(32), None) == rcb.OK
    assert lib.refcache_f8_linear_gelu_backward(empty(32), weight(), 0, empty(64), P, 64, empty(64), None) == rcb.OK


def test_unknown_form_by_name(lib):
    with pytest.raises(ValueError, match="form"):
        rcb._gelu_form("sigmoid")


def test_weight_grad_workspace_is_bounded(lib):
    """The values of one panel of x in bf16 (256 MB, or 256 columns), and parts of dw for no more tiles than the GPU takes at a time."""
    f = lib.refcache_f8_weight_grad_bytes
    for r in (1, 320, 4608, 1 << 20, (1 << 31) - 600):
        for n, k in ((16, 16), (272, 208), (1024, 1024), (16384, 4096)):
            panel = max(256 << 20, r * min(k, 256) * 2)
            assert min(r * min(k, 256) * 2, panel) <= f(r, n, k) <= panel + 256 + 76 * 256 * 256 * 4
    assert f(0, 16, 16) == f(-1, 16, 16) == 0 and f(4, 8, 16) == 0 and f(4, 16, 24) == 0
