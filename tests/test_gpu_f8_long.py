"""The 8-bit calls on tensors of more than 2^31 elements: the last rows must be what a call on these rows alone gives."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rc

pytestmark = pytest.mark.gpu
BF16, U8 = torch.bfloat16, torch.uint8


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    yield
    torch.cuda.empty_cache()
    assert rc.status() == rc.OK, rc.last_error()


def rnd(seed, *s):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(s, generator=g, device="cuda", dtype=BF16)


def tail(f, rows):
    return f.codes[-rows:].view(U8), f.scales.view(U8)[-rows:]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_rows_and_products():
    """140000 rows of 16400: 2.3e9 elements, and outputs as long."""
    rows, width, last = 140000, 16400, 1000
    x = rnd(0, rows, width)
    x8, end8 = rc.f8_quantize(x), rc.f8_quantize(x[-last:])
    assert same(tail(x8, last), tail(end8, last))
    w = rc.f8_quantize_weight(rnd(1, width, 64))  # y [rows, width] from 64 columns, and back
    a, enda = rc.f8_quantize(x[:, :64]), rc.f8_quantize(x[-last:, :64])
    del x
    y, end = torch.empty(rows, width, dtype=BF16, device="cuda"), torch.empty(last, width, dtype=BF16, device="cuda")
    rc.f8_linear(a, w, y)
    rc.f8_linear(enda, w, end)
    assert torch.equal(y[-last:], end)
    del y
    z, endz = torch.empty(rows, 64, dtype=BF16, device="cuda"), torch.empty(last, 64, dtype=BF16, device="cuda")
    rc.f8_linear(x8, w, z, transposed=True)
    rc.f8_linear(end8, w, endz, transposed=True)
    # (the two calls take the sums apart differently: within a rounding of each)
    assert (z[-last:].double() - endz.double()).abs().max() <= 2.0 ** -7 * endz.double().abs().max()
    g, u = rc.F8Rows(rows, width), rc.F8Rows(rows, width)
    rc.f8_linear_gelu(a, w, g, u, form="tanh")
    eg, eu = rc.F8Rows(last, width), rc.F8Rows(last, width)
    rc.f8_linear_gelu(enda, w, eg, eu, form="tanh")
    assert same(tail(g, last), tail(eg, last)) and same(tail(u, last), tail(eu, last))


def test_weight_gradient():
    """dw of more than 2^31 elements, and of rows of x and dy of as many, in panels."""
    n, k = 46400, 46400
    x, dy = rnd(0, 64, k), rnd(1, 64, n)
    dw = torch.empty(n, k, dtype=BF16, device="cuda")
    rc.f8_weight_grad(dy, rc.f8_quantize(x), dw)
    end = torch.empty(400, k, dtype=BF16, device="cuda")
    rc.f8_weight_grad(dy[:, -400:], rc.f8_quantize(x), end)
    assert torch.equal(dw[-400:], end)
    del dw, x, dy
    rows = 140000
    x, dy = rnd(2, rows, 16400), rnd(3, rows, 16)
    dw = torch.empty(16, 16400, device="cuda")
    x8 = rc.f8_quantize(x)
    rc.f8_weight_grad(dy, x8, dw)
    del x
    v = x8.codes[:, -16:].double() * torch.exp2(x8.scales.view(U8)[:, -1:].double() - 127)
    want = dy.double().t() @ v
    assert ((dw[:, -16:].double() - want).norm() / want.norm()) <= 1e-5
