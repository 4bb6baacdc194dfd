"""Linear layers in 8 bits against their definitions in 64 bits: the 8-bit form bit for bit, products within the rounding
of their sums and of the result."""
import math

import pytest
import torch

import f8_reference as ref
from paper_2608_21229_gb300 import refcache as rc

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *s, gain=1.0, dtype=BF16):
    return (torch.randn(s, generator=g, device="cuda") * gain).to(dtype)


def uneven(g, r, c, gain=1.0):
    """Rows whose blocks have scales of their own."""
    x = torch.randn(r, c, generator=g, device="cuda")
    return (x * torch.exp2(torch.randint(-12, 6, (r, 1), generator=g, device="cuda").float()) *
            torch.exp(torch.randn(c, generator=g, device="cuda")) * gain).to(BF16)


def apart(t, pad=24):
    """The same values in rows that lie apart."""
    big = torch.full((t.shape[0], t.shape[1] + pad), -777.0, dtype=t.dtype, device=t.device)
    v = big[:, 8:8 + t.shape[1]]
    v.copy_(t)
    return v


def sums(terms):
    """The bound of a sum of products in fp32 by the tensor core or by FMAs: `terms` additions, each off by at most one unit
    in the last place (2^-23: the tensor core may truncate) of a partial sum, which is at most the sum of magnitudes."""
    return (terms + 2) * 2.0 ** -23


def check(got, want, mag, terms, half_step):
    """|got - want| within the sum's bound (`mag`: the sum of magnitudes) and half a step of the result's type."""
    tol = sums(terms) * mag * (1 + half_step) + half_step * want.abs() + 2.0 ** -133
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all()
    bad = off > tol
    assert not bad.any(), (int(bad.sum()), off[bad][:4].tolist(), tol[bad][:4].tolist())
    # the bound counts every addition at its worst; the typical error is far below it
    if want.numel() >= 1000 and want.norm() > 0:
        assert (off.norm() / want.norm()) <= half_step + 2.0 ** -14


def near_form(f, want, delta):
    """That an F8Rows holds the 8-bit form of values within `delta` of `want`: each scale's power of two is the smallest
    for a largest value within delta, each value within half a step of its code, 2^-4 of itself or 2^-10 of the scale."""
    r, c = want.shape
    b = f.scales.view(torch.uint8).long()
    s = torch.exp2(b.double() - 127)
    pad = torch.zeros(r, b.shape[1] * 128, dtype=torch.float64, device=want.device)
    lo, hi = pad.clone(), pad.clone()
    lo[:, :c], hi[:, :c] = (want.abs() - delta).clamp(min=0), want.abs() + delta
    lo, hi = lo.view(r, -1, 128).amax(2), hi.view(r, -1, 128).amax(2)
    fits = (s * 448 >= lo) & ((s * 224 < hi) | (b == 1) | ((lo == 0) & (b == 127)))
    assert fits.all(), (b[~fits][:4], lo[~fits][:4], hi[~fits][:4])
    off = (ref.meant(f) - want).abs()
    tol = delta * (1 + 2.0 ** -4) + torch.maximum(want.abs() * 2.0 ** -4, ref.spread(b, want.shape).double().sub(137).exp2())
    assert (off <= tol * (1 + 1e-12)).all(), float((off - tol).max())


def check_tiles(f):
    """The tensor cores' copies of the scales, as the header says where each lies."""
    for tiles, scales, height, tall in ((f._tiles, f.scales, f.codes.shape[0], 128 if hasattr(f, "codes_t") else 1),) + (
            ((f._tiles_t, f.scales_t, f.codes_t.shape[0], 128),) if hasattr(f, "codes_t") else ()):
        b = scales.view(torch.uint8)
        r, j = torch.arange(height, device="cuda")[:, None], torch.arange(b.shape[1], device="cuda")[None]
        at = 512 * ((j // 4) * -(-height // 128) + r // 128) + 16 * (r % 32) + 4 * (r // 32 % 4) + j % 4
        assert torch.equal(tiles.flatten()[at], b.repeat_interleave(tall, 0)[:height])


# ---------------------------------------------------------------- the 8-bit form
@pytest.mark.parametrize("r, c", [(1, 16), (1, 4096), (3, 128), (5, 144), (33, 272), (257, 1808), (2, 8208), (1000, 256),
                                  (40000, 16), (30001, 272), (10000, 1040), (5, 512), (6, 528)])
def test_rows_bit_for_bit(r, c):
    g = gen(r * 10007 + c)
    x = uneven(g, r, c)
    x[0, : c // 2] = 0
    if r > 2:
        x[2] = 0
        x[1, 0] = 448 * 2.0 ** 3  # a largest value on the border
    for src in (x, apart(x)):
        f = rc.f8_quantize(src)
        codes, b = ref.form(x)
        assert torch.equal(f.scales.view(torch.uint8).long(), b)
        assert torch.equal(f.codes.double(), codes)
        check_tiles(f)


def test_rows_at_the_borders_of_scales_and_codes():
    """Largest values next to 448 times powers of two, every bf16 exponent, and halves between codes."""
    g = gen(5)
    e = torch.arange(-133, 128, device="cuda").float()
    x = torch.randn(len(e) * 4, 128, generator=g, device="cuda", dtype=torch.float64).clamp(-3.4, 3.4)
    near = torch.tensor([1.0, 1.75, 1.7578125, 1.7421875], dtype=torch.float64, device="cuda")
    x = torch.exp2(e.double()).repeat_interleave(4)[:, None] * x.abs().clamp(max=1.0) * torch.sign(x)
    x[:, 7] = torch.exp2(e.double()).repeat_interleave(4) * near.repeat(len(e))
    x = x.to(BF16)
    x = x[torch.isfinite(x).all(1)].contiguous()
    f = rc.f8_quantize(x)
    codes, b = ref.form(x)
    assert torch.equal(f.scales.view(torch.uint8).long(), b)
    # (below 2^-126 x / 2^-126 is taken of what is left of a subnormal, which fp32 holds exactly)
    assert torch.equal(f.codes.double(), codes)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_block_with_a_value_that_is_not_finite_is_nan(bad):
    x = randn(gen(1), 4, 400)
    x[1, 130] = bad
    f = rc.f8_quantize(x)
    codes, b = ref.form(x)
    got = ref.meant(f)
    assert torch.isnan(got[1, 128:256]).all() and torch.isfinite(got[1, :128]).all() and torch.isfinite(got[1, 256:]).all()
    assert torch.isfinite(got[[0, 2, 3]]).all()
    assert torch.equal(f.scales.view(torch.uint8).long(), b)
    w = rc.f8_quantize_weight(randn(gen(2), 272, 400))
    y = torch.empty(4, 272, dtype=BF16, device="cuda")
    rc.f8_linear(f, w, y)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[[0, 2, 3]]).all()
    dw = torch.empty(32, 400, device="cuda")
    rc.f8_weight_grad(randn(gen(3), 4, 32), f, dw)
    assert torch.isnan(dw[:, 128:256]).all() and torch.isfinite(dw[:, :128]).all() and torch.isfinite(dw[:, 256:]).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("n, k", [(16, 16), (128, 128), (144, 400), (400, 144), (1040, 2064), (256, 4096)])
def test_weight_bit_for_bit(n, k, dtype):
    g = gen(n + k)
    w = (torch.randn(n, k, generator=g, device="cuda") * torch.exp(torch.randn(k, generator=g, device="cuda"))).to(dtype)
    w[: n // 2, : k // 2] *= 1e-3
    f = rc.f8_quantize_weight(w)
    codes, b = ref.form(w, 128)
    assert torch.equal(f.scales.view(torch.uint8).long(), b) and torch.equal(f.scales_t.view(torch.uint8).long(), b.t())
    assert torch.equal(f.codes.double(), codes) and torch.equal(f.codes_t.double(), codes.t())
    check_tiles(f)


def test_one_orientation_alone():
    w = randn(gen(9), 144, 272)
    f, both = rc.F8Weight(144, 272), rc.f8_quantize_weight(w)
    f.c.codes_t = f.c.scales_t = f.c.tiles_t = None
    f.codes_t.view(torch.uint8).fill_(3)
    rc.f8_quantize_weight(w, f)
    assert torch.equal(f.codes.view(torch.uint8), both.codes.view(torch.uint8)) and (f.codes_t.view(torch.uint8) == 3).all()
    with pytest.raises(rc.RefCacheError):
        rc.f8_linear(rc.f8_quantize(randn(gen(1), 4, 144)), f, torch.empty(4, 272, dtype=BF16, device="cuda"), transposed=True)


# ---------------------------------------------------------------- products
SHAPES = [  # rows, n, k
    (1, 16, 16), (1, 4096, 1024), (2, 128, 4096), (3, 2576, 528), (7, 48, 2064), (16, 512, 512), (17, 400, 144), (31, 1040, 272),
    (64, 256, 8208), (65, 272, 1040), (100, 768, 256), (129, 128, 128), (255, 272, 640), (256, 256, 512), (257, 528, 528), (320, 768, 256),
    (333, 272, 208), (513, 1296, 784), (777, 2064, 400), (1024, 1024, 1024), (2100, 3600, 656),
    (200, 2064, 8208),  # few rows in two tiles, columns split
    (1777, 8240, 784),  # tiles of 192 columns
    (1500, 4112, 2064)]  # several rounds of tiles, and of 1024 rows


@pytest.mark.parametrize("r, n, k", SHAPES)
@pytest.mark.parametrize("transposed", [False, True], ids=["xwT", "xw"])
def test_linear(r, n, k, transposed):
    g = gen(r + 3 * n + 7 * k)
    inn, out = (n, k) if transposed else (k, n)
    x, w = rc.f8_quantize(uneven(g, r, inn)), rc.f8_quantize_weight(randn(g, n, k, gain=inn ** -0.5))
    bias = [None, randn(g, out), randn(g, out, dtype=F32)][r % 3]
    y = apart(torch.zeros(r, out, dtype=BF16, device="cuda")) if r % 2 else torch.empty(r, out, dtype=BF16, device="cuda")
    rc.f8_linear(x, w, y, bias=bias, transposed=transposed)
    assert rc.status() == rc.OK
    a, b = ref.meant(x), ref.meant(w)
    b = b if transposed else b.t()
    want, mag = a @ b, a.abs() @ b.abs()
    if bias is not None:
        want, mag = want + bias.double(), mag + bias.double().abs()
    check(y, want, mag, inn + 1, 2.0 ** -8)
    if r % 2:
        base = y._base
        assert (base[:, :8] == -777).all() and (base[:, 8 + out:] == -777).all()
    again = torch.empty(r, out, dtype=BF16, device="cuda")
    rc.f8_linear(x, w, again, bias=bias, transposed=transposed)
    assert torch.equal(again.view(torch.int16), y.contiguous().view(torch.int16))


@pytest.mark.parametrize("form", ["erf", "tanh"])
@pytest.mark.parametrize("r, n, k", SHAPES)
def test_linear_gelu(r, n, k, form):
    g = gen(r + 5 * n + 11 * k)
    x, w = rc.f8_quantize(randn(g, r, k, gain=2.0)), rc.f8_quantize_weight(randn(g, n, k, gain=k ** -0.5))
    bias = [randn(g, n, dtype=F32), None, randn(g, n)][r % 3]
    a, u8 = rc.F8Rows(r, n), rc.F8Rows(r, n)
    rc.f8_linear_gelu(x, w, a, u8, bias=bias, form=form)
    assert rc.status() == rc.OK
    vx, vw = ref.meant(x), ref.meant(w)
    u, mag = vx @ vw.t(), vx.abs() @ vw.abs().t()
    if bias is not None:
        u, mag = u + bias.double(), mag + bias.double().abs()
    delta = sums(k + 1) * mag
    near_form(u8, u, delta)
    # the derivative is at most 1.13.  The tail of the normal distribution and the logistic function are off by some units of
    # fp32 (a fit within 1.3e-7, 2^-22 for each of exp2 and the reciprocal, ten roundings: below 2^-19 together) and by what the rounding of their
    # exponents, u^2 / 2 log2 e or (1.6 |u| + 0.072 |u|^3) log2 e, does: three times 2^-24 of them times ln 2
    g = ref.gelu(u, form).abs()
    near_form(a, ref.gelu(u, form), 1.13 * delta + g * (2.0 ** -19 + 2.0 ** -22 * (u.abs() + u * u + u.abs() ** 3 / 8)) + 2.0 ** -126)
    check_tiles(u8)
    check_tiles(a)
    only = rc.F8Rows(r, n)
    rc.f8_linear_gelu(x, w, only, bias=bias, form=form)
    assert torch.equal(only.codes.view(torch.uint8), a.codes.view(torch.uint8))
    assert torch.equal(only.scales.view(torch.uint8), a.scales.view(torch.uint8))


@pytest.mark.parametrize("form", ["erf", "tanh"])
@pytest.mark.parametrize("r, n, k", SHAPES)
def test_linear_gelu_backward(r, n, k, form):
    """Here w is [n, k]: dy has n columns, u and du have k."""
    g = gen(r + 13 * n + 17 * k)
    dy, w = rc.f8_quantize(uneven(g, r, n, 1e-3)), rc.f8_quantize_weight(randn(g, n, k, gain=n ** -0.5))
    u8 = rc.f8_quantize(randn(g, r, k, gain=1.5))
    du = apart(torch.zeros(r, k, dtype=BF16, device="cuda")) if r % 2 else torch.empty(r, k, dtype=BF16, device="cuda")
    du8 = rc.F8Rows(r, k)
    rc.f8_linear_gelu_backward(dy, w, u8, du, du8, form=form)
    assert rc.status() == rc.OK
    a, b, u = ref.meant(dy), ref.meant(w), ref.meant(u8)
    slope = ref.gelu_grad(u, form)
    da, mag = a @ b, a.abs() @ b.abs()
    want = da * slope
    # the slope's own error: its terms are at most 1.2, the derivative's argument has fp32's relative error, and its rate of
    # change times u stays below 3
    delta = sums(n) * mag * slope.abs() + da.abs() * 2.0 ** -19
    off = (du.double() - want).abs()
    assert (off <= delta * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs() + 2.0 ** -133).all()
    near_form(du8, want, delta + 2.0 ** -140)
    check_tiles(du8)
    alone, alone8 = torch.empty(r, k, dtype=BF16, device="cuda"), rc.F8Rows(r, k)
    rc.f8_linear_gelu_backward(dy, w, u8, alone, None, form=form)
    rc.f8_linear_gelu_backward(dy, w, u8, None, alone8, form=form)
    assert torch.equal(alone, du) and torch.equal(alone8.codes.view(torch.uint8), du8.codes.view(torch.uint8))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("r, n, k", SHAPES + [(4099, 144, 272), (9000, 256, 256), (20608, 32, 528)])
def test_weight_grad(r, n, k, dtype):
    g = gen(r + 19 * n + 23 * k)
    dy, x = uneven(g, r, n, 1e-3), rc.f8_quantize(uneven(g, r, k))
    add = randn(g, n, k, gain=1e-2, dtype=dtype) if r % 2 else None
    db = torch.empty(n, device="cuda") if r % 3 == 0 or r == 4099 else None
    dw = torch.empty(n, k, dtype=dtype, device="cuda")
    rc.f8_weight_grad(apart(dy) if r % 4 == 1 else dy, x, dw, add=add, d_bias=db)
    assert rc.status() == rc.OK
    v = ref.meant(x)
    want, mag = dy.double().t() @ v, dy.double().abs().t() @ v.abs()
    if add is not None:
        want, mag = want + add.double(), mag + add.double().abs()
    check(dw, want, mag, r + 1, 2.0 ** -24 if dtype is F32 else 2.0 ** -8)
    if db is not None:
        check(db, dy.double().sum(0), dy.double().abs().sum(0), r, 2.0 ** -24)
    if add is not None:  # in place
        rc.f8_weight_grad(dy, x, add, add=add)
        assert torch.equal(add, dw)


def test_weight_grad_of_large_and_small_scales():
    """Rows whose scales lie anywhere between 2^-100 and 2^100, beside ordinary ones and alone."""
    g = gen(31)
    for spread in ((-100, 100), (8, 100), (-100, -60), (7, 9)):
        e = torch.randint(spread[0], spread[1], (200, 1), generator=g, device="cuda").float()
        x = rc.f8_quantize((torch.randn(200, 272, generator=g, device="cuda") * torch.exp2(e)).to(BF16))
        dy = (torch.randn(200, 144, generator=g, device="cuda") * torch.exp2(-e)).to(BF16)
        dw = torch.empty(144, 272, device="cuda")
        rc.f8_weight_grad(dy, x, dw)
        v = ref.meant(x)
        check(dw, dy.double().t() @ v, dy.double().abs().t() @ v.abs(), 201, 2.0 ** -24)


def test_weight_grad_by_differences():
    """L(w) = sum of dy times (x w^T), in 64 bits, has dw as its slope (it is linear in w: any step will do)."""
    g = gen(77)
    dy, x = randn(g, 100, 48), rc.f8_quantize(randn(g, 100, 272))
    dw = torch.empty(48, 272, device="cuda")
    rc.f8_weight_grad(dy, x, dw)
    w, v = torch.randn(48, 272, dtype=torch.float64, device="cuda"), ref.meant(x)
    loss = lambda w: (dy.double() * (v @ w.t())).sum()  # noqa: E731
    for n, k in ((0, 0), (47, 271), (13, 130)):
        e = torch.zeros_like(w)
        e[n, k] = 0.5
        slope = loss(w + e) - loss(w - e)
        assert abs(float(dw[n, k]) - float(slope)) <= sums(100) * float((dy.double().abs().t() @ v.abs())[n, k]) + 1e-9


@pytest.mark.parametrize("form", ["erf", "tanh"])
def test_gelu_gradient_by_differences(form):
    """du is the slope of sum(da gelu(u)) at u, central differences in 64 bits (error h^2 / 6 times a third derivative below 2)."""
    g = gen(78)
    dy, w, u8 = rc.f8_quantize(randn(g, 20, 64)), rc.f8_quantize_weight(randn(g, 64, 144, gain=0.1)), rc.f8_quantize(randn(g, 20, 144, gain=2.0))
    du = torch.empty(20, 144, dtype=BF16, device="cuda")
    rc.f8_linear_gelu_backward(dy, w, u8, du, form=form)
    da, u, h = ref.meant(dy) @ ref.meant(w), ref.meant(u8), 1e-4
    slope = da * (ref.gelu(u + h, form) - ref.gelu(u - h, form)) / (2 * h)
    mag = ref.meant(dy).abs() @ ref.meant(w).abs()
    assert ((du.double() - slope).abs() <= 2.0 ** -8 * slope.abs() + sums(64) * mag * 1.2 + da.abs() * (2.0 ** -19 + 1e-8)).all()


@pytest.mark.parametrize("form", ["erf", "tanh"])
def test_gelu_gradient_at_zeros_of_both_signs(form):
    u = torch.zeros(4, 128, dtype=BF16, device="cuda")
    u[1] = -0.0
    u[2, ::2], u[3, 1::2] = -0.0, 2.0 ** -120
    dy, w = rc.f8_quantize(torch.ones(4, 16, dtype=BF16, device="cuda")), rc.f8_quantize_weight(torch.ones(16, 128, dtype=BF16, device="cuda"))
    du = torch.empty(4, 128, dtype=BF16, device="cuda")
    rc.f8_linear_gelu_backward(dy, w, rc.f8_quantize(u), du, form=form)
    assert (du == 8.0).all()


@pytest.mark.parametrize("form", ["erf", "tanh"])
def test_gelu_gradient_far_from_zero(form):
    """The gradient is 1 above and 0 below, to the largest values that the 8-bit form holds, whose squares are infinite."""
    u = torch.empty(6, 128, dtype=BF16, device="cuda")
    for i, size in enumerate((16.0, 2.0 ** 20, 2.0 ** 63, 2.0 ** 64, 2.0 ** 100, 448 * 2.0 ** 118)):
        u[i, ::2], u[i, 1::2] = size, -size
    dy, w = rc.f8_quantize(torch.ones(6, 16, dtype=BF16, device="cuda")), rc.f8_quantize_weight(torch.ones(16, 128, dtype=BF16, device="cuda"))
    du = torch.empty(6, 128, dtype=BF16, device="cuda")
    rc.f8_linear_gelu_backward(dy, w, rc.f8_quantize(u), du, form=form)
    assert (du[:, ::2] == 16.0).all() and (du[:, 1::2].abs() <= 1e-20).all()


# On 76 CTA pairs: 80, 95, 102 and 184 tiles of 256 columns, of which the last 4 and 19 may go in four pieces each, the last 26 and 32 in two.
PIECES = [(1025, 4096, 1040), (1025, 4848, 528), (1300, 4112, 272), (1801, 5872, 272)]


@pytest.mark.parametrize("r, n, k", PIECES)
def test_tiles_in_pieces(r, n, k):
    test_linear(r, n, k, False)
    test_linear(r, k, n, True)
    test_linear_gelu(r, n, k, "erf")
    test_linear_gelu_backward(r, k, n, "tanh")


@pytest.mark.parametrize("r, n, k", [(3001, 8208, 16), (2990, 2576, 640), (2990, 2576, 656), (5000, 4112, 144)])
def test_many_rows_of_few_columns(r, n, k):
    test_linear(r, n, k, False)
    test_linear(r, k, n, True)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("r, n, k", [(700, 4848, 1040), (260, 4112, 1296), (1100, 4848, 1040)])
def test_weight_grad_tiles_in_halves(r, n, k, dtype):
    """On 76 CTA pairs: 95 and 102 tiles, of which the last 19 and 26 go in halves; one and two sets of 1024 rows."""
    test_weight_grad(r, n, k, dtype)


# ---------------------------------------------------------------- no rows, streams, graphs
def test_without_rows():
    x, w = rc.F8Rows(0, 64), rc.f8_quantize_weight(randn(gen(1), 32, 64))
    rc.f8_quantize(torch.empty(0, 64, dtype=BF16, device="cuda"), x)
    rc.f8_linear(x, w, torch.empty(0, 32, dtype=BF16, device="cuda"))
    rc.f8_linear_gelu(x, w, rc.F8Rows(0, 32), rc.F8Rows(0, 32))
    rc.f8_linear_gelu_backward(rc.F8Rows(0, 32), w, x, torch.empty(0, 64, dtype=BF16, device="cuda"), rc.F8Rows(0, 64))
    dw, db, add = torch.full((32, 64), 7.0, device="cuda"), torch.full((32,), 7.0, device="cuda"), randn(gen(2), 32, 64, dtype=F32)
    dy = torch.empty(0, 32, dtype=BF16, device="cuda")
    rc.f8_weight_grad(dy, x, dw, d_bias=db)
    assert (dw == 0).all() and (db == 0).all()
    rc.f8_weight_grad(dy, x, dw, add=add)
    assert torch.equal(dw, add)


def mlp(x, w1, w2, b1, b2, target_grad, form="tanh", stream=None):
    """A block's MLP forwards and backwards as a training step runs it: every checkpoint in 8 bits."""
    r, c, h = x.shape[0], w1.in_width, w1.out_width
    kw = {"stream": stream}
    x8 = rc.f8_quantize(x, rc.F8Rows(r, c), **kw)
    a8, u8 = rc.F8Rows(r, h), rc.F8Rows(r, h)
    rc.f8_linear_gelu(x8, w1, a8, u8, bias=b1, form=form, **kw)
    y = torch.empty(r, c, dtype=BF16, device="cuda")
    rc.f8_linear(a8, w2, y, bias=b2, **kw)
    g = {n: torch.empty(s, device="cuda") for n, s in (("dw1", (h, c)), ("dw2", (c, h)), ("db1", (h,)), ("db2", (c,)))}
    dy8 = rc.f8_quantize(target_grad, rc.F8Rows(r, c), **kw)
    du, du8, dx = torch.empty(r, h, dtype=BF16, device="cuda"), rc.F8Rows(r, h), torch.empty(r, c, dtype=BF16, device="cuda")
    rc.f8_linear_gelu_backward(dy8, w2, u8, du, du8, form=form, **kw)
    rc.f8_weight_grad(target_grad, a8, g["dw2"], d_bias=g["db2"], **kw)
    rc.f8_linear(du8, w1, dx, transposed=True, **kw)
    rc.f8_weight_grad(du, x8, g["dw1"], d_bias=g["db1"], **kw)
    return {"y": y, "dx": dx, **g}


def mlp_inputs(r=333, c=272, h=1040, seed=0):
    g = gen(seed)
    w = [randn(g, h, c, gain=c ** -0.5, dtype=F32), randn(g, c, h, gain=h ** -0.5, dtype=F32)]
    return randn(g, r, c), w, [randn(g, h, gain=0.1), randn(g, c, gain=0.1)], randn(g, r, c, gain=1e-2)


@pytest.mark.parametrize("form", ["erf", "tanh"])
def test_an_mlp_in_8_bits(form):
    """The calls together, against the same MLP in 64 bits without any rounding.  A code is off by at most 2^-4 of its value,
    uniformly about 2^-4 / sqrt(3) / 1.4 of it (0.026); a product of two such factors by 0.037 of itself, terms with errors of
    their own, so that a sum of them has the same share: 0.037.  y goes through two such products one after the other (0.05),
    dx through two and the slope at a rounded u (curvature times 0.026 u: below 0.03), dw1 through those of dx's first and x;
    so no result is off by more than 0.1 of its norm."""
    x, w, b, dy = mlp_inputs()
    got = mlp(x, rc.f8_quantize_weight(w[0]), rc.f8_quantize_weight(w[1]), b[0], b[1], dy, form)
    leaf = [t.double().requires_grad_() for t in (x, w[0], w[1], b[0], b[1])]
    u = leaf[0] @ leaf[1].t() + leaf[3]
    y = ref.gelu(u, form) @ leaf[2].t() + leaf[4]
    grads = torch.autograd.grad(y, leaf, dy.double())
    want = dict(zip(("dx", "dw1", "dw2", "db1", "db2"), grads), y=y.detach())
    for n, v in want.items():
        rel = float((got[n].double() - v).norm() / v.norm())
        assert rel <= 0.1, (n, rel)
    assert rc.status() == rc.OK


def test_other_streams_and_graph_replay():
    x, w, b, dy = mlp_inputs(seed=4)
    w1, w2 = (rc.f8_quantize_weight(t) for t in w)
    want = mlp(x, w1, w2, b[0], b[1], dy)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = mlp(x, w1, w2, b[0], b[1], dy)
    s.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want)
    xin, dyin = x.clone(), dy.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mlp(xin, w1, w2, b[0], b[1], dyin)
    for seed in (5, 6):
        x2, _, _, dy2 = mlp_inputs(seed=seed)
        want = mlp(x2, w1, w2, b[0], b[1], dy2)
        xin.copy_(x2)
        dyin.copy_(dy2)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[n]) for n in want)
    assert rc.status() == rc.OK


def test_two_streams_at_once():
    """Calls that overlap share nothing."""
    sets = [mlp_inputs(r, seed=r) for r in (200, 777)]
    ws = [[rc.f8_quantize_weight(t) for t in s[1]] for s in sets]
    want = [mlp(s[0], w[0], w[1], *s[2], s[3]) for s, w in zip(sets, ws)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(10):
        for i, (s, w) in enumerate(zip(sets, ws)):
            with torch.cuda.stream(streams[i]):
                got[i].append(mlp(s[0], w[0], w[1], *s[2], s[3]))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(g[n], want[i][n]) for n in g)


def test_results_made_on_another_stream():
    """A call with a stream allocates what it returns for that stream."""
    x = randn(gen(8), 300, 272)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    want, w = rc.f8_quantize(x), randn(gen(9), 144, 272)
    want_w = rc.f8_quantize_weight(w)
    torch.cuda.synchronize()
    for _ in range(20):
        torch.empty(300 * 272, dtype=torch.uint8, device="cuda").fill_(7)  # freed, and perhaps still being written
        f, fw = rc.f8_quantize(x, stream=s), rc.f8_quantize_weight(w, stream=s)
        s.synchronize()
        assert torch.equal(f.codes.view(torch.uint8), want.codes.view(torch.uint8)) and torch.equal(f._mem[:, :3], want._mem[:, :3])
        assert torch.equal(fw.codes_t.view(torch.uint8), want_w.codes_t.view(torch.uint8))


def test_weight_grad_in_panels():
    """x's values are taken in panels of columns where all of them would need too much memory: 36000 rows of 4096 in two.  Few
    columns of dy, and every 50th column of dw against 64 bits."""
    g = gen(41)
    dy, x = randn(g, 36000, 48), rc.f8_quantize(uneven(g, 36000, 4096))
    dw, add = torch.empty(48, 4096, device="cuda"), randn(g, 48, 4096, dtype=F32)
    assert rc.load().refcache_f8_weight_grad_bytes(36000, 48, 4096) < 36000 * 4096 * 2
    rc.f8_weight_grad(dy, x, dw, add=add)
    v = x.codes[:, ::50].double() * torch.exp2(x.scales.view(torch.uint8).double() - 127).repeat_interleave(128, 1)[:, ::50]
    check(dw[:, ::50], dy.double().t() @ v + add[:, ::50].double(), dy.double().abs().t() @ v.abs() + add[:, ::50].double().abs(), 36001, 2.0 ** -24)
    assert rc.status() == rc.OK


def test_binding_refusals():
    g = gen(3)
    x, w = rc.f8_quantize(randn(g, 4, 64)), rc.f8_quantize_weight(randn(g, 32, 64))
    y = torch.empty(4, 32, dtype=BF16, device="cuda")
    with pytest.raises(ValueError, match="F8Rows"):
        rc.f8_linear(x.codes, w, y)
    with pytest.raises(ValueError, match="y"):
        rc.f8_linear(x, w, y.float())
    with pytest.raises(ValueError, match="y"):
        rc.f8_linear(x, w, y.t())
    with pytest.raises(ValueError, match="contiguous"):
        rc.f8_linear(x, w, torch.empty(32, 4, dtype=BF16, device="cuda").t())
    with pytest.raises(ValueError, match="bias"):
        rc.f8_linear(x, w, y, bias=torch.zeros(16, device="cuda"))
    with pytest.raises(rc.RefCacheError):
        rc.f8_linear(x, w, torch.empty(4, 64, dtype=BF16, device="cuda"), transposed=True)
    with pytest.raises(rc.RefCacheError):
        rc.f8_quantize(torch.empty(4, 24, dtype=BF16, device="cuda"))
    with pytest.raises(ValueError, match="GPU"):
        rc.f8_quantize(torch.empty(4, 32, dtype=BF16))
    with pytest.raises(ValueError, match="dw"):
        rc.f8_weight_grad(y, x, torch.empty(32, 32, device="cuda"))
    with pytest.raises(ValueError, match="add"):
        rc.f8_weight_grad(y, x, torch.empty(32, 64, device="cuda"), add=torch.empty(32, 64, dtype=BF16, device="cuda"))
    with pytest.raises(ValueError, match="dy"):
        rc.f8_weight_grad(y[:3], x, torch.empty(32, 64, device="cuda"))
    with pytest.raises(rc.RefCacheError):  # rows on top of each other
        rc.f8_weight_grad(y[:1].expand(4, 32), x, torch.empty(32, 64, device="cuda"))
