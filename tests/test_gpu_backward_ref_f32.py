"""Gradients of cached rows held in float32, which a sum over many steps of one cache needs: in bf16 each step's call
rounds the sum again, and what is below 2^-9 of it is lost."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

from test_gpu_backward import KERNELS, Case, Ref, default_kernel  # noqa: F401  (a fixture)
from test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
CASES = [
    (3, 128, [(13, 40, 217, 301), (0, 0, 130, 127), (7, 0, 0, 65), (5, 3, 254, 0)], "beyond"),
    (2, 128, [(13, 40, 217, 301), (128, 1, 127, 129), (0, 5, 60, 257)], "beyond_alt"),
    (2, 64, [(77, 30, 153, 204), (13, 40, 77, 102), (64, 0, 1, 64)], "beyond_alt"),
    (3, 64, [(0, 64, 193, 385), (0, 0, 64, 1)], "isolated"),
    (2, 64, [(i % 9, i % 5, 3 * i % 40, 7 * i % 31) for i in range(75)], "beyond"),  # more requests than one launch's list holds
]


def inputs(c):
    o, lse = c.step_ref(Ref())
    return o.to(BF16), lse.float()


def f32_refs(c, fill=float("nan")):
    return [torch.full(c.ref_shape, fill, device="cuda") for _ in range(2)]


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"d{c[1]}x{len(c[2])}{c[3]}")
def test_float32_is_what_bf16_is_rounded_from(case, kernel):
    c = Case(*case)
    rcb.set_kernel(kernel)
    o, lse = inputs(c)
    half = c.step_backward(o, lse)
    single = c.step_backward(o, lse, into=f32_refs(c))
    for n, t in half.items():
        assert torch.equal(single[n].to(BF16), t), n
    assert (single["dk_ref"] != half["dk_ref"].float()).float().mean() > 0.5  # (not rounded on its way)
    # added to what is there: one rounding of the sum, one of the product with the scale
    into = [torch.randn(c.ref_shape, device="cuda", generator=torch.Generator(device="cuda")) for _ in range(2)]
    held = [t.clone() for t in into]
    again = c.step_backward(o, lse, into=into, accumulate=True)
    for n, h in zip(("dk_ref", "dv_ref"), held):
        size = h.double().abs() + single[n].double().abs()
        assert ((again[n].double() - h.double() - single[n].double()).abs() <= 2.0 ** -23 * size).all(), n
    # into the prefill's gradients: the same floats as bf16 gives where they are the same, and the definition's elsewhere
    ref = Ref()
    o, lse = c.build_ref(ref)
    o, lse = o.to(BF16), lse.float()
    refs = [half["dk_ref"], half["dv_ref"]]
    for a, b in zip(c.build_backward(o, lse, *refs).values(), c.build_backward(o, lse, *(t.float() for t in refs)).values()):
        assert torch.equal(a, b)
    add = {}
    for n, h in zip(("dk", "dv"), held):
        add[n] = torch.zeros(c.static[0].shape, device="cuda")
        add[n][c.cached] = h
    for n, t in c.build_backward(o, lse, *held).items():
        ref.check(n, t, add.get(n))


@pytest.mark.parametrize("dim", [64, 128])
def test_many_steps_are_summed_without_loss(dim):
    """200 steps: the sum in fp32 is within its 200 roundings of the sum of the steps' gradients."""
    c = Case(2, dim, [(8, 16, 200, 300)])
    o, lse = inputs(c)
    one = c.step_backward(o, lse, into=f32_refs(c))
    n, into = 200, f32_refs(c, 0.0)
    for _ in range(n):
        c.step_backward(o, lse, into=into, accumulate=True)
    for name, t in zip(("dk_ref", "dv_ref"), into):
        want = n * one[name].double()
        assert ((t.double() - want).abs() <= n * 2.0 ** -24 * want.abs() + 1e-30).all(), name


@pytest.mark.parametrize("kernel", KERNELS)
def test_no_live_rows_at_all(kernel):
    rcb.set_kernel(kernel)
    c = Case(2, 128, [(7, 0, 0, 300), (0, 0, 0, 1)])
    o, lse = torch.empty(0, 2, 128, dtype=BF16, device="cuda"), torch.empty(0, 2, device="cuda")
    g = c.step_backward(o, lse, into=f32_refs(c))
    assert (g["dk_ref"] == 0).all() and (g["dv_ref"] == 0).all()
    into = [torch.randn(c.ref_shape, device="cuda") for _ in range(2)]
    held = [t.clone() for t in into]
    c.step_backward(o, lse, into=into, accumulate=True)
    assert all(torch.equal(a, b) for a, b in zip(into, held))


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("case", CASES[1:3], ids=lambda c: f"d{c[1]}")
def test_nothing_beside_them_is_written(case, kernel):
    c = Case(*case)
    rcb.set_kernel(kernel)
    o, lse = inputs(c)
    g = [Guarded(c.ref_shape, F32) for _ in range(2)]
    c.step_backward(o, lse, into=[x.t for x in g])
    for x in g:
        x.check("float32 gradient of the cached rows")


def test_refusals():
    c = Case(2, 128, [(4, 8, 20, 30)])
    o, lse = inputs(c)
    q, k, v, do = c.live
    out = [torch.empty_like(q) for _ in range(3)]
    f, h = torch.zeros(c.ref_shape, device="cuda"), torch.zeros(c.ref_shape, dtype=BF16, device="cuda")
    for dk, dv, match in ((f, h, "dv_ref"), (h, f, "dv_ref"), (f, None, "dv_ref"), (None, f, "dk_ref"), (f, f[:5], "dv_ref"), (f.double(), f, "dk_ref"),
                          (f, f.cpu(), "dv_ref")):
        with pytest.raises(ValueError, match=match):
            c.cache.step_backward(0, q, k, v, o, lse, do, *out, dk_ref=dk, dv_ref=dv)
    with pytest.raises(ValueError, match="contiguous"):
        c.cache.step_backward(0, q, k, v, o, lse, do, *out, dk_ref=f, dv_ref=f.transpose(1, 2).contiguous().transpose(1, 2))
