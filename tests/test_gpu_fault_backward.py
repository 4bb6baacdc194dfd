"""Waits of the gradient kernels that run out, without a GPU fault: on the host's request a producer stops before one of
its loads, in the first or the second CTA of each pair, so that the teardown finds the pair's loads apart in one ring or
several.  The kernels report it, free their tensor memory and return, and the next call is correct."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

from test_gpu_backward import Case, Ref

pytestmark = pytest.mark.gpu

KEYS, SECOND = 1 << 8, 1 << 9


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kernel", [0, KEYS], ids=["queries", "keys"])
def test_gradient_wait_timeouts_are_reported_and_the_context_survives(dim, kernel):
    rcb.load()
    rcb.set_kernel("tcgen05")
    c = Case(24, dim, [(16, 40, 700, 900)])  # 72 and 168 items of 13 and 6 tiles: some pairs have two, whose loads go on
    o, lse = c.step_ref(Ref())
    o, lse = o.to(torch.bfloat16), lse.float()
    want = c.step_backward(o, lse)
    torch.cuda.synchronize()
    assert rcb.status() == rcb.OK and c.cache.status() == rcb.OK
    for second in (0, SECOND):
        for load in (1, 2, 3, 4, 5, 6, 7, 9, 12, 13):
            old = rcb.set_wait_timeout_ns(20_000_000)  # 20 ms
            try:
                rcb.debug_skip_first_load(load | kernel | second)
                c.step_backward(o, lse)
                assert c.cache.status() == rcb.ERR_TIMEOUT, (second, load)
                assert rcb.status() == rcb.ERR_TIMEOUT and "wait ran out" in rcb.last_error()
                assert c.cache.status() == rcb.OK and rcb.status() == rcb.OK  # cleared
            finally:
                rcb.debug_skip_first_load(0)
                rcb.set_wait_timeout_ns(old)
            got = c.step_backward(o, lse)
            for n in want:
                assert torch.equal(got[n], want[n]), (second, load, n)
    assert rcb.status() == rcb.OK
