"""Waits of the 8-bit products that run out, without a GPU fault: on the host's request a producer stops before one of its
loads, in the first or the second CTA of each pair (or cluster), so that the teardown finds their loads apart.  The
kernels report it, free their tensor memory and return, and the next call is correct."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rc

pytestmark = pytest.mark.gpu

SECOND = 1 << 9
BF16 = torch.bfloat16


def rnd(seed, *s):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(s, generator=g, device="cuda")


def linear():
    x, w = rc.f8_quantize(rnd(0, 3000, 1040).to(BF16)), rc.f8_quantize_weight(rnd(1, 3600, 1040))

    def call():
        y = torch.empty(3000, 3600, dtype=BF16, device="cuda")
        rc.f8_linear(x, w, y)
        return y

    return call


def few():
    x, w = rc.f8_quantize(rnd(0, 20, 4112).to(BF16)), rc.f8_quantize_weight(rnd(1, 1040, 4112))

    def call():
        y = torch.empty(20, 1040, dtype=BF16, device="cuda")
        rc.f8_linear(x, w, y)
        return y

    return call


def gelu():
    x, w = rc.f8_quantize(rnd(0, 2000, 784).to(BF16)), rc.f8_quantize_weight(rnd(1, 4112, 784))

    def call():
        a = rc.F8Rows(2000, 4112)
        rc.f8_linear_gelu(x, w, a)
        return a.codes.view(torch.uint8)

    return call


def pieces():
    """80 tiles of nine loads each, so that on 76 pairs the last four are shared out in pieces of nine loads."""
    x, w = rc.f8_quantize(rnd(0, 1025, 1040).to(BF16)), rc.f8_quantize_weight(rnd(1, 4096, 1040))

    def call():
        y = torch.empty(1025, 4096, dtype=BF16, device="cuda")
        rc.f8_linear(x, w, y)
        return y

    return call


def halves():
    """95 tiles of eleven loads each, so that on 76 pairs the last 19 are shared out in halves of eleven loads."""
    x, dy = rc.f8_quantize(rnd(0, 700, 1040).to(BF16)), rnd(1, 700, 4848).to(BF16)

    def call():
        dw = torch.empty(4848, 1040, device="cuda")
        rc.f8_weight_grad(dy, x, dw)
        return dw

    return call


def weight_grad():
    x, dy = rc.f8_quantize(rnd(0, 1300, 2064).to(BF16)), rnd(1, 1300, 4112).to(BF16)

    def call():
        dw = torch.empty(4112, 2064, device="cuda")
        rc.f8_weight_grad(dy, x, dw)
        return dw

    return call


@pytest.mark.parametrize("make", [linear, few, gelu, weight_grad], ids=lambda f: f.__name__)
def test_wait_timeouts_are_reported_and_the_context_survives(make):
    check_timeouts(make(), (1, 2, 3, 5, 6, 7, 8))


def test_wait_timeouts_in_pieces_of_tiles():
    check_timeouts(pieces(), (9, 10, 11, 12, 13, 14, 16, 18))


def test_wait_timeouts_in_halves_of_tiles():
    check_timeouts(halves(), (10, 11, 12, 13, 15, 17, 18, 22))


def check_timeouts(call, loads):
    want = call()
    torch.cuda.synchronize()
    assert rc.status() == rc.OK
    for second in (0, SECOND):
        for load in loads:
            old = rc.set_wait_timeout_ns(20_000_000)  # 20 ms
            try:
                rc.debug_skip_first_load(load | second)
                call()
                assert rc.status() == rc.ERR_TIMEOUT and "wait ran out" in rc.last_error(), (second, load)
                assert rc.status() == rc.OK  # cleared
            finally:
                rc.debug_skip_first_load(0)
                rc.set_wait_timeout_ns(old)
            assert torch.equal(call(), want), (second, load)
    assert rc.status() == rc.OK
