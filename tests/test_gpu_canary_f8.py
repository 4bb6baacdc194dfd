"""Guard bytes around every buffer that the 8-bit calls write, their workspaces among them: nothing is written beside an
output, no element of one is left out, and no input changes.  Sizes end inside tiles, and rows lie apart."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rc

from test_gpu_canary import Guarded
from test_gpu_canary_block import Inputs, works  # noqa: F401

pytestmark = pytest.mark.gpu
BF16, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


def rnd(seed, *s, gain=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(s, generator=g, device="cuda") * gain


class Form:
    """An F8Rows between guards."""

    def __init__(self, rows, width):
        self.f = rc.F8Rows(rows, width)
        self.g = [Guarded(t.shape, U8) for t in (self.f.codes, self.f._mem, self.f._tiles)]
        self.f.c.codes, self.f.c.scales, self.f.c.tiles = (g.t.data_ptr() for g in self.g)

    def check(self, want):
        """Guards, and that all is there: the codes and scales of a call on memory of another content (a code may be the pattern)."""
        for g, n in zip(self.g, ("codes", "scales", "tiles")):
            g.check(n, written=False)
        blocks = want.scales.shape[1]
        assert torch.equal(self.g[0].t, want.codes.view(U8)) and torch.equal(self.g[1].t[:, :blocks], want._mem[:, :blocks])


def blank(rows, width):
    f = rc.F8Rows(rows, width)
    for t in (f.codes.view(U8), f._mem, f._tiles):
        t.fill_(0)
    return f


def kept(f):
    return [t for t in (f.codes.view(U8), f._mem, f._tiles)]


@pytest.mark.parametrize("rows, width", [(1, 16), (37, 272), (300, 1040), (1000, 528), (5, 4112)])
def test_quantize(rows, width, works):  # noqa: F811
    x = rnd(rows, rows, width + 8).to(BF16)[:, :width]
    k, f = Inputs(x), Form(rows, width)
    rc.f8_quantize(x, f.f)
    torch.cuda.synchronize()
    f.check(rc.f8_quantize(x, blank(rows, width)))
    k.check()


@pytest.mark.parametrize("n, k", [(16, 16), (144, 272), (272, 144), (400, 1040)])
def test_quantize_weight(n, k, works):  # noqa: F811
    w, f = rnd(n, n, k), rc.F8Weight(n, k)
    fields = ("codes", "scales", "tiles", "codes_t", "scales_t", "tiles_t")
    g = [Guarded(t.shape, U8) for t in (f.codes, f._mem, f._tiles, f.codes_t, f._mem_t, f._tiles_t)]
    for name, x in zip(fields, g):
        setattr(f.c, name, x.t.data_ptr())
    kin = Inputs(w)
    rc.f8_quantize_weight(w, f)
    torch.cuda.synchronize()
    for name, x in zip(fields, g):
        x.check(name, written=False)
    want = rc.F8Weight(n, k)
    for t in (want.codes, want.codes_t, want._mem, want._mem_t):
        t.view(U8).fill_(0)
    rc.f8_quantize_weight(w, want)
    assert torch.equal(g[0].t, want.codes.view(U8)) and torch.equal(g[3].t, want.codes_t.view(U8))
    kin.check()


@pytest.mark.parametrize("rows, n, k", [(1, 16, 16), (20, 1040, 4112), (130, 272, 1040), (200, 2064, 8208), (300, 528, 272), (1777, 8240, 784), (2100, 3600, 656)])
def test_products(rows, n, k, works):  # noqa: F811
    x, w = rc.f8_quantize(rnd(0, rows, k).to(BF16)), rc.f8_quantize_weight(rnd(1, n, k, gain=k ** -0.5))
    dy, u = rc.f8_quantize(rnd(2, rows, n).to(BF16)), rc.f8_quantize(rnd(3, rows, k).to(BF16))
    bias = rnd(4, n)
    kin = Inputs(*kept(x), w.codes.view(U8), w.codes_t.view(U8), w._mem, w._mem_t, w._tiles, w._tiles_t, *kept(dy), *kept(u), bias)
    y, yt, du = Guarded((rows, n), BF16), Guarded((rows, k), BF16), Guarded((rows, k), BF16)
    a, u8, du8 = Form(rows, n), Form(rows, n), Form(rows, k)
    rc.f8_linear(x, w, y.t, bias=bias)
    rc.f8_linear(dy, w, yt.t, transposed=True)
    rc.f8_linear_gelu(x, w, a.f, u8.f, bias=bias, form="tanh")
    rc.f8_linear_gelu_backward(dy, w, u, du.t, du8.f, form="erf")
    torch.cuda.synchronize()
    for name, g in (("y", y), ("yt", yt), ("du", du)):
        g.check(name)
    wa, wu, wdu = blank(rows, n), blank(rows, n), blank(rows, k)
    rc.f8_linear_gelu(x, w, wa, wu, bias=bias, form="tanh")
    rc.f8_linear_gelu_backward(dy, w, u, None, wdu, form="erf")
    for f, want in ((a, wa), (u8, wu), (du8, wdu)):
        f.check(want)
    kin.check()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("rows, n, k", [(1, 16, 16), (100, 144, 272), (700, 400, 1040), (4099, 144, 272), (1300, 4112, 2064)])
def test_weight_grad(rows, n, k, dtype, works):  # noqa: F811
    x, dy, add = rc.f8_quantize(rnd(0, rows, k).to(BF16)), rnd(1, rows, n + 24).to(BF16)[:, 8:8 + n], rnd(2, n, k).to(dtype)
    kin = Inputs(*kept(x), dy, add)
    dw, db = Guarded((n, k), dtype), Guarded((n,), F32)
    rc.f8_weight_grad(dy, x, dw.t, add=add, d_bias=db.t)
    torch.cuda.synchronize()
    dw.check("dw")
    db.check("d_bias")
    kin.check()
