"""The sums of the 8-bit products: how far the tensor cores' additions, which cut off what does not fit, may take them from 64
bits.  A sum goes through tensor memory for 16384 columns of x (1024 rows of a weight gradient) at most, so that what is cut off
does not grow with longer ones."""
import pytest
import torch

import f8_reference as ref
import test_gpu_f8 as f8
from paper_2608_21229_gb300 import refcache as rc

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

# rows, columns of the result, columns that are summed: on 76 CTA pairs tiles of 64, 128 (one and two rounds), 192 and 256 columns, the last
# ones in pieces of 64 and 128; few rows: the columns split eight ways, of which a CTA has one or several sets of 16384
LONG = [(2600, 272, 16400), (3000, 272, 33040), (5000, 784, 16400), (1300, 1552, 16400), (1025, 4112, 16400), (1300, 4848, 16400),
        (20, 272, 140016), (130, 400, 135184), (64, 1040, 262160)]


@pytest.mark.parametrize("r, n, k", LONG)
def test_long_rows(r, n, k):
    f8.test_linear(r, n, k, False)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("r, n, k", [LONG[i] for i in (1, 4, 7)])
def test_long_rows_transposed(r, n, k):
    f8.test_linear(r, k, n, True)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("form", ["erf", "tanh"])
@pytest.mark.parametrize("r, n, k", [LONG[i] for i in (1, 4, 6)])
def test_long_rows_gelu(r, n, k, form):
    f8.test_linear_gelu(r, n, k, form)
    f8.test_linear_gelu_backward(r, k, n, form)
    torch.cuda.empty_cache()


def operands(r, n, k, one_sign):
    g = f8.gen(k + r)
    x, w = torch.randn(r, k, generator=g, device="cuda"), torch.randn(n, k, generator=g, device="cuda") * k ** -0.5
    if one_sign:
        x, w = x.abs(), w.abs()
    return x.to(BF16), w


def linear_error(r, n, k, one_sign):
    """The error's norm over y's, of eight rows: what is left of y beside a bias of -y, which bf16 rounds by 2^-8 of itself."""
    x, w = operands(r, n, k, one_sign)
    x8, w8 = rc.f8_quantize(x), rc.f8_quantize_weight(w)
    rows = list(range(0, r, max(1, r // 8)))
    a = ref.value(x8.codes[rows], x8.scales.view(torch.uint8)[rows])
    y = a @ ref.meant(w8).t()
    out, off = torch.empty(r, n, dtype=BF16, device="cuda"), []
    for i, row in enumerate(rows):
        bias = (-y[i]).float()
        rc.f8_linear(x8, w8, out, bias=bias)
        off.append(out[row].double() - (y[i] + bias.double()))
    assert rc.status() == rc.OK
    return float(torch.stack(off).norm() / y.norm())


@pytest.mark.parametrize("one_sign, at_4096, at_16384", [(False, 3e-7, 1.5e-6), (True, 2e-6, 1.2e-5)])
def test_linear_sums(one_sign, at_4096, at_16384):
    """The bounds of the header, at each width's most additions in a row (tiles, and few rows in one CTA's columns)."""
    for r, n, k, most in ((4608, 1024, 4096, at_4096), (2, 24576, 4096, at_4096), (4608, 1024, 16384, at_16384)):
        e = linear_error(r, n, k, one_sign)
        assert e <= most, (r, n, k, e)


@pytest.mark.parametrize("one_sign", [False, True])
@pytest.mark.parametrize("r, n, k", [(4608, 512, 65536), (2, 24576, 65536), (1000, 272, 262144), (120, 1040, 262160), (2, 128, 1 << 20)])
def test_longer_sums_are_as_exact(r, n, k, one_sign):
    """Sets of 16384 columns are added up to nearest: a sum of up to 64 of them, each with the error of one, is off by that share
    of itself, and by 2^-24 of a partial sum for each addition, as a random walk of at most 64 steps 8 * 2^-24 = 4.8e-7."""
    one = linear_error(4608, 512, 16384, one_sign)
    e = linear_error(r, n, k, one_sign)
    torch.cuda.empty_cache()
    assert e <= 1.05 * one + 5e-7, (e, one)


@pytest.mark.parametrize("one_sign", [False, True])
@pytest.mark.parametrize("r, n, k", [(4608, 528, 1040), (9000, 272, 528), (20608, 144, 272)])
def test_weight_grad_sums(r, n, k, one_sign):
    """64 additions in tensor memory between two to nearest: 64 additions of a product make 2.1e-7 (1024 columns of the 8-bit product above), here
    of 16 rows each twice that, and the additions of 5 to 21 sets a few times 2^-24."""
    g = f8.gen(r)
    x, dy = torch.randn(r, k, generator=g, device="cuda"), torch.randn(r, n, generator=g, device="cuda")
    if one_sign:
        x, dy = x.abs(), dy.abs()
    x8, dy, dw = rc.f8_quantize(x.to(BF16)), dy.to(BF16), torch.empty(n, k, device="cuda")
    rc.f8_weight_grad(dy, x8, dw)
    want = dy.double().t() @ ref.meant(x8)
    assert float((dw.double() - want).norm() / want.norm()) <= 1e-6
