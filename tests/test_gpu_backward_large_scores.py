"""Gradients at scores of hundreds, where P is nearly one-hot and a score and its row's log-sum-exp cancel, against 64
bits.  The bounds are test_gpu_backward's, with the allowance for scores in proportion to them: a score is a sum of products
in fp32, right to 2^-21 of the sum of their sizes, as are its product with scale log2 e and the log-sum-exp in fp32."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

import test_gpu_backward as tb
from test_gpu_backward import KERNELS, Case, Ref, default_kernel  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("gain", [40.0, 200.0])
def test_large_scores(dim, kernel, gain, monkeypatch):
    c = Case(2, dim, [(4, 8, 150, 200), (0, 3, 128, 129)], gain=gain)
    rcb.set_kernel(kernel)
    sizes = lambda q, k: (q.double().abs().transpose(0, 1) @ k.double().abs().transpose(0, 1).transpose(1, 2)).max().item() * c.scale  # noqa: E731
    q, k = c.live[:2]
    most = max(sizes(q, k), sizes(q, c.static[1]), sizes(*c.static[:2]))
    assert gain * 4 < most < gain * 64
    monkeypatch.setattr(tb, "F", most * 2.0 ** -21)
    ref = Ref()
    o, lse = c.step_ref(ref)
    assert lse.abs().max() > gain
    for n, t in c.step_backward(o.to(torch.bfloat16), lse.float()).items():
        assert t.abs().max() > 0.1, n
        ref.check(n, t)
    ref = Ref()
    o, lse = c.build_ref(ref)
    for n, t in c.build_backward(o.to(torch.bfloat16), lse.float()).items():
        ref.check(n, t)
