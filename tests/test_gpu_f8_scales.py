"""That every block of columns is multiplied with its own scales, of x and of the weight, however often the slots that hold
them are used again."""
import pytest
import torch

import f8_reference as ref
from paper_2608_21229_gb300 import refcache as rc
from test_gpu_canary_f8 import test_products as guarded_products
from test_gpu_canary import Guarded  # noqa: F401
from test_gpu_canary_block import works  # noqa: F401
from test_gpu_f8 import check, gen

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def scaled(g, rows, k, e, tall):
    """Values whose scales differ by 2^e[j] from block to block of columns, and by some more from one `tall` rows to the next."""
    x = torch.randn(rows, k, generator=g, device="cuda").clamp(-3, 3)
    own = torch.randint(-3, 4, (-(-rows // tall), len(e)), generator=g, device="cuda")
    return x * torch.exp2(ref.spread(own + e, (rows, k), tall).float())


# rows, columns of y, columns of x.  On 152 SMs: few rows with x's columns in one piece (5, 8 and 19 groups of scales a CTA, the last one short), in
# three, four and seven (5 and 6 groups); tiles (33 groups a tile in one round; 5 in two rounds, the last in pieces)
SHAPES = [(2, 19904, 2192), (2, 24576, 4096), (5, 22000, 9232), (17, 12304, 8208), (16, 7776, 8208), (300, 2624, 10080), (2, 16, 16896), (130, 16, 16448),
          (3000, 528, 16400), (1025, 4112, 2192)]


@pytest.mark.parametrize("r, n, k", SHAPES)
def test_linear(r, n, k):
    """Blocks of x as much larger as the weight's are smaller, so that each is as much of y as the others: a block taken with
    another's scale would be off by powers of two."""
    g = gen(r + n + k)
    e = torch.randint(-20, 21, (-(-k // 128),), generator=g, device="cuda")
    x8 = rc.f8_quantize(scaled(g, r, k, e, 1).to(BF16))
    w8 = rc.f8_quantize_weight(scaled(g, n, k, -e, 128))
    assert len(x8.scales.view(torch.uint8).unique()) > 10 and len(w8.scales.view(torch.uint8).unique()) > 10
    y = torch.empty(r, n, dtype=BF16, device="cuda")
    rc.f8_linear(x8, w8, y)
    assert rc.status() == rc.OK
    a, b = ref.meant(x8), ref.meant(w8).t()
    check(y, a @ b, a.abs() @ b.abs(), k + 1, 2.0 ** -8)


@pytest.mark.parametrize("rows, n, k", [(2, 19904, 2192), (16, 7776, 8208), (130, 16, 16448), (20, 272, 140016)])
def test_nothing_beside_the_results(rows, n, k, works):  # noqa: F811
    guarded_products(rows, n, k, works)
