"""The 8-bit form at the upper end of bf16.  From 248 * 2^120 on a row's scale is 2^120 and its largest code 256: 2^128, above
every finite bf16 and fp32.  What reads values back takes that as bf16's largest, 255 * 2^120, so that finite rows stay finite."""
import pytest
import torch

import f8_reference as ref
from paper_2608_21229_gb300 import refcache as rc

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
LARGEST = 255 * 2.0 ** 120
SIZES = [LARGEST, 248 * 2.0 ** 120, 247 * 2.0 ** 120, 224 * 2.0 ** 120, 448 * 2.0 ** 119]


def rows(width):
    """Rows whose largest values are SIZES, of both signs, beside small ones, zeros and, in a block of their own, ordinary ones."""
    x = torch.zeros(len(SIZES), width, dtype=BF16, device="cuda")
    for i, size in enumerate(SIZES):
        x[i, ::4], x[i, 1::4], x[i, 2::4] = size, -size, 1.5 * 2.0 ** 113
    x[:, 128:256] = torch.linspace(-3, 3, 128, device="cuda", dtype=BF16)[: x[:, 128:256].shape[1]]
    return x


def meant(f):
    return ref.meant(f).clamp(-LARGEST, LARGEST)


@pytest.mark.parametrize("n, k", [(16, 400), (144, 128), (528, 1040)])
def test_weight_grad(n, k):
    x = rc.f8_quantize(rows(k))
    assert (x.scales.view(torch.uint8)[:, 0] == torch.tensor([247, 247, 247, 246, 246], device="cuda")).all() and (x.codes[:2, 0].float() == 256).all()
    dy = (torch.randn(len(SIZES), n, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda") * 2.0 ** -20).to(BF16)
    dy[:, ::3] = 0
    dw = torch.empty(n, k, device="cuda")
    rc.f8_weight_grad(dy, x, dw)
    assert torch.isfinite(dw).all() and (dw[::3] == 0).all()
    v = meant(x)
    want, mag = dy.double().t() @ v, dy.double().abs().t() @ v.abs()
    # six additions and a rounding, each off by 2^-23 of the magnitudes at most
    assert ((dw.double() - want).abs() <= (len(SIZES) + 2) * 2.0 ** -23 * mag).all()


def test_blocks_that_are_not_finite_stay_nan():
    x = rows(400)
    x[1, 0], x[2, 300] = float("inf"), float("nan")
    dy = torch.full((len(SIZES), 16), 2.0 ** -20, dtype=BF16, device="cuda")
    dw = torch.empty(16, 400, device="cuda")
    rc.f8_weight_grad(dy, rc.f8_quantize(x), dw)
    assert torch.isnan(dw[:, :128]).all() and torch.isfinite(dw[:, 128:256]).all() and torch.isnan(dw[:, 256:384]).all() and torch.isfinite(dw[:, 384:]).all()


@pytest.mark.parametrize("form", ["erf", "tanh"])
@pytest.mark.parametrize("copies, n, k", [(1, 2064, 128), (1, 4112, 272), (1, 16, 144), (400, 272, 272)])  # few rows (two), tiles (two)
def test_gelu_gradient(copies, n, k, form):
    """The gradient is 1 above and 0 below; dy w is the same in every column."""
    u = rows(k)
    u[:, 128:256] = u[:, :128][:, : u[:, 128:256].shape[1]]
    u = u.repeat(copies, 1)
    dy, w = torch.ones(len(u), n, dtype=BF16, device="cuda"), torch.ones(n, k, dtype=BF16, device="cuda")
    du, du8 = torch.empty(len(u), k, dtype=BF16, device="cuda"), rc.F8Rows(len(u), k)
    rc.f8_linear_gelu_backward(rc.f8_quantize(dy), rc.f8_quantize_weight(w), rc.f8_quantize(u), du, du8, form=form)
    assert torch.equal(du[u > 0], torch.full_like(du[u > 0], n)) and (du[u < 0] == 0).all()
    # at zero half of dy w, off by the slope's own error, 2^-19 of dy w, and half a step: 4112 / 2 lies in the middle of two bf16 values
    assert ((du[u == 0].double() - 0.5 * n).abs() <= 2.0 ** -8 * 0.5 * n + 2.0 ** -19 * n).all()
    assert torch.isfinite(ref.meant(du8)).all()


@pytest.mark.parametrize("copies, n, k", [(1, 272, 4112), (300, 272, 272)])
def test_products_are_of_what_the_codes_stand_for(copies, n, k):
    """A scale is applied by the tensor core, where 2^128 is no bound of a factor."""
    x = rows(k).repeat(copies, 1)
    x[:, 4:] = 0
    w = torch.full((n, k), 2.0 ** -12, dtype=BF16, device="cuda")
    w[:, 1] = 0
    y = torch.empty(len(x), n, dtype=BF16, device="cuda")
    x8, w8 = rc.f8_quantize(x), rc.f8_quantize_weight(w)
    rc.f8_linear(x8, w8, y)
    want = ref.meant(x8) @ ref.meant(w8).t()
    assert torch.isfinite(y).all() and ((y.double() - want).abs() <= 2.0 ** -7 * want.abs()).all()
