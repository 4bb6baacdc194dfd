"""Waits of the 8-bit products that run out behind the first use of what they use again: the scales' slots of few rows, and the
tensor memory of sums that go on in registers (from the 129th load of a CTA on)."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rc
from test_gpu_f8_fault import BF16, check_timeouts, rnd

pytestmark = pytest.mark.gpu


def linear(r, n, k):
    x, w = rc.f8_quantize(rnd(0, r, k).to(BF16)), rc.f8_quantize_weight(rnd(1, n, k))

    def call():
        y = torch.empty(r, n, dtype=BF16, device="cuda")
        rc.f8_linear(x, w, y)
        return y

    return call


def gelu(r, n, k):
    x, w = rc.f8_quantize(rnd(0, r, k).to(BF16)), rc.f8_quantize_weight(rnd(1, n, k))

    def call():
        a = rc.F8Rows(r, n)
        rc.f8_linear_gelu(x, w, a)
        return a.codes.view(torch.uint8)

    return call


def test_few_rows_behind_the_first_wrap_of_the_scales():
    """17 x 12304 x 8208 on 152 SMs: split three ways, 24, 24 and 17 loads and six and five groups of scales a CTA, in four slots."""
    check_timeouts(linear(17, 12304, 8208), (16, 17, 18, 20, 21, 24))


@pytest.mark.parametrize("make, r, n", [(linear, 2600, 272), (gelu, 5000, 784)])
def test_long_rows_in_tiles(make, r, n):
    check_timeouts(make(r, n, 33040), (127, 128, 129, 130, 134, 160, 255))


@pytest.mark.parametrize("make", [linear, gelu])
def test_long_rows_few(make):
    check_timeouts(make(64, 272, 262160), (127, 128, 129, 130, 134, 160, 255))
