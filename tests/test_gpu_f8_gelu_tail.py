"""The GELU and its gradient where it is nearly nothing: a block of nothing but arguments far below zero has a scale of its own, in
which 1 - erf or 1 - tanh would leave no digits.  The distribution's tail and the logistic function are held in relative terms."""
import pytest
import torch

import f8_reference as ref
import test_gpu_f8 as f8
from paper_2608_21229_gb300 import refcache as rc

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# Blocks' centres; half a unit to each side stays where the values are normal in fp32: u phi(u) at -12.9 is 3e-37, its tanh form at -9.4 3e-33
CENTRES = {"erf": [-3.5, -5.0, -7.0, -9.0, -11.0, -12.4], "tanh": [-3.5, -4.5, -5.5, -6.5, -7.5, -8.9]}
SHAPES = [(700, 16), (2100, 144), (3, 4112), (20, 4112), (130, 16448)]  # rows and columns of x: in tiles (two), few rows (three)


def gelu(u, form):
    """u phi(u) in 64 bits with phi from erfc, or as the logistic function: 1 + erf and 1 + tanh have no digits left here."""
    if form == "erf":
        return 0.5 * u * torch.special.erfc(-u * 0.5 ** 0.5)
    return u * torch.sigmoid(2 * (2 / torch.pi) ** 0.5 * (u + 0.044715 * u ** 3))


def gelu_grad(u, form):
    """phi(u) + u phi'(u)."""
    if form == "erf":
        return 0.5 * torch.special.erfc(-u * 0.5 ** 0.5) + u * torch.exp(-0.5 * u * u) * (0.5 / torch.pi) ** 0.5
    a = 2 * (2 / torch.pi) ** 0.5
    z = a * (u + 0.044715 * u ** 3)
    return torch.sigmoid(z) + u * torch.sigmoid(z) * torch.sigmoid(-z) * a * (1 + 3 * 0.044715 * u * u)


def test_the_definitions_here():
    """Where neither loses digits they are torch's."""
    u = torch.linspace(-4, 4, 1001, dtype=torch.float64)
    for form in CENTRES:
        assert (gelu(u, form) - ref.gelu(u, form)).abs().max() < 1e-14 and (gelu_grad(u, form) - ref.gelu_grad(u, form)).abs().max() < 1e-14


def relative(u):
    """The relative error of the GELU and of its derivative's parts, as test_gpu_f8.py derives it: some units of fp32, below 2^-19, and the
    rounding of the exponents u^2 / 2 or 1.6 |u| + 0.072 |u|^3, three times 2^-24 of them."""
    return 2.0 ** -19 + 2.0 ** -22 * (u.abs() + u * u + u.abs() ** 3 / 8)


def arguments(form, seed, rows=None):
    """One row, or `rows` of them, of a block around each centre."""
    c = torch.tensor(CENTRES[form], device="cuda").repeat_interleave(128)
    shape = c.shape if rows is None else (rows, len(c))
    return c + torch.rand(shape, generator=f8.gen(seed), device="cuda") - 0.5


def tail_share(form):
    """The smallest value's block is far below 1: its scale is of these values alone."""
    return gelu(torch.tensor(CENTRES[form][-1] + 0.5, dtype=torch.float64), form).abs().item()


@pytest.mark.parametrize("form", ["erf", "tanh"])
@pytest.mark.parametrize("r, k", SHAPES)
def test_forward(r, k, form):
    assert 0 < tail_share(form) < 1e-20
    n = 128 * len(CENTRES[form])
    g = f8.gen(r + k)
    # products that add up to 1e-3 at most: u is the bias and a little more, in every row another
    x = rc.f8_quantize(f8.randn(g, r, k))
    w = rc.f8_quantize_weight(f8.randn(g, n, k, gain=2e-4 * k ** -0.5))
    bias = arguments(form, k)
    a, u8 = rc.F8Rows(r, n), rc.F8Rows(r, n)
    rc.f8_linear_gelu(x, w, a, u8, bias=bias, form=form)
    assert rc.status() == rc.OK
    vx, vw = ref.meant(x), ref.meant(w)
    u, mag = vx @ vw.t() + bias.double(), vx.abs() @ vw.abs().t()
    delta = f8.sums(k) * mag + 2.0 ** -24 * u.abs()  # the products' sum, and the bias rounded in
    want = gelu(u, form)
    # |d gelu / du| over |gelu| is below 1 / |u| + the exponent's slope, |u| or 1.6 + 0.215 u^2: so much of the value is what u is off by
    steep = 1 / u.abs() + torch.maximum(u.abs(), 1.6 + 0.215 * u * u) + 1
    tol = (relative(u) + steep * delta) * want.abs()
    f8.near_form(u8, u, delta)
    f8.near_form(a, want, tol)
    # A code differs from that of 64 bits where a border lies within the tolerance of the value: two borders at least 2^-4 of it apart
    codes, b = ref.form(want)
    same = ref.spread((a.scales.view(torch.uint8).long() == b).long(), want.shape) == 1
    differ = ((a.codes.double() != codes) & same).double().mean().item()
    assert same.double().mean() >= 1 - 1e-2 and differ <= 32 * (tol / want.abs()).mean().item() + 8 / want.numel(), differ


@pytest.mark.parametrize("form", ["erf", "tanh"])
@pytest.mark.parametrize("r, n", SHAPES)
def test_gradient(r, n, form):
    """dy w is 1 in every column."""
    k = 128 * len(CENTRES[form])
    u8 = rc.f8_quantize(arguments(form, n, r).to(BF16))
    dy, w = torch.zeros(r, n, dtype=BF16, device="cuda"), torch.zeros(n, k, dtype=BF16, device="cuda")
    dy[:, 5], w[5] = 1, 1
    du, du8 = torch.empty(r, k, dtype=BF16, device="cuda"), rc.F8Rows(r, k)
    rc.f8_linear_gelu_backward(rc.f8_quantize(dy), rc.f8_quantize_weight(w), u8, du, du8, form=form)
    assert rc.status() == rc.OK
    u = ref.meant(u8)
    want = gelu_grad(u, form)
    # the parts phi(u) and u times the density have opposite signs: the second is at least nine times the first below -3
    tol = 1.25 * relative(u) * want.abs()
    assert ((du.double() - want).abs() <= tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()).all()
    f8.near_form(du8, want, tol)
