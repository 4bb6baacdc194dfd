"""clip_gradients under an infinite bound: the norm alone, in place and out of place, whatever the norm is."""
import math

import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("special", [2.0, math.inf, -math.inf, math.nan, 3e38], ids=str)
@pytest.mark.parametrize("out32", [False, True])
def test_an_infinite_bound_leaves_the_values(special, out32):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    grads = [torch.randn(n, generator=gen, device="cuda").to(dt)[1:] for n, dt in ((300, torch.bfloat16), (40001, torch.float32))]
    grads[1][7] = special
    before = [t.clone() for t in grads]
    want = math.sqrt(sum(t.double().square().sum().item() for t in grads))
    if abs(special) == 3e38:
        want = math.inf  # (as documented: its square is beyond fp32)
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))  # noqa: E731
    outs = [torch.full(t.shape, 7.0, dtype=torch.float32 if out32 else t.dtype, device="cuda") for t in grads]
    for norm in (rcb.clip_gradients(grads, math.inf, out=outs), rcb.clip_gradients(grads, math.inf)):
        if math.isfinite(want):
            assert abs(norm.item() - want) <= 1e-5 * want
        else:
            assert norm.isnan() if math.isnan(want) else norm.item() == want
    for g, o, b in zip(grads, outs, before):
        assert same(g, b) and torch.equal(o.isnan(), b.isnan())
        assert torch.equal(o.double().nan_to_num(nan=0.5), b.double().nan_to_num(nan=0.5))
    assert rcb.status() == rcb.OK
