"""gated_norm and its gradient on as many rows as a call takes, 2^31 - 513: the last block's rows end past 2^31."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
ROWS, WIDTH, LAST = (1 << 31) - 513, 8, 3000


def test_the_last_rows_of_the_longest_call():
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB of device memory")
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    some = torch.randn(1 << 20, WIDTH, generator=g, device="cuda").to(BF16)
    x = torch.empty(ROWS, WIDTH, dtype=BF16, device="cuda")
    for at in range(0, ROWS, len(some)):  # (random rows of all of it would take longer than the calls)
        x[at:at + len(some)] = some[:ROWS - at]
    x[-LAST:] = torch.randn(LAST, WIDTH, generator=g, device="cuda").to(BF16)
    scale = torch.randn(2, WIDTH, generator=g, device="cuda")
    out = torch.full_like(x, float("nan"))
    tail, want = x[-LAST:].clone(), torch.empty(LAST, WIDTH, dtype=BF16, device="cuda")
    cu, alone, kw = [0, ROWS - LAST, ROWS], [0, LAST], dict(scale=scale[1:].clone())
    rcb.gated_norm(cu, x, out, scale=scale)
    rcb.gated_norm(alone, tail, want, **kw)
    assert torch.equal(out[-LAST:], want) and not out[::4099].isnan().any()
    out.fill_(float("nan"))
    sums = torch.full((2, WIDTH), float("nan"), device="cuda")
    rcb.gated_norm_backward(cu, x, x, out, scale=scale, d_shift=sums)
    rcb.gated_norm_backward(alone, tail, tail, want, **kw)
    assert torch.equal(out[-LAST:], want) and not out[::4099].isnan().any()
    exact = tail.double().sum(0)
    assert ((sums[1].double() - exact).abs() <= LAST * 2.0 ** -23 * tail.double().abs().sum(0)).all()
    assert torch.isfinite(sums).all() and rcb.status() == rcb.OK
