"""gated_norm's gradient with requests that have no rows: what their gate and scale hold reaches nothing."""
import math

import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

from test_gpu_block_ops import BF16, NormCase

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,width,mdtype", [
    ([40, 0, 70, 0], 264, torch.float32),  # many slots a request: one request after the other
    ([0, 3, 0, 9, 4, 0] + [2] * 20, 136, BF16),  # few
    ([3, 0] * 40 + [0], 64, torch.float32),  # two launches, the second's first request without rows
], ids=lambda x: str(len(x)) if isinstance(x, list) else None)
def test_requests_without_rows_add_nothing(lens, width, mdtype):
    c = NormCase(lens, width, "layer", "rms", mdtype, True)
    empty = torch.tensor([n == 0 for n in lens], device="cuda")
    runs = []
    for fill in (1.0, math.nan, math.inf):
        mods = {n: c.mods[n].clone() for n in ("gate", "scale")}
        for t in mods.values():
            t[empty] = fill
        f32 = lambda *s: torch.full(s, math.nan, device="cuda")  # noqa: E731
        got = {"d_gate": f32(c.B, width), "d_scale": f32(c.B, width), "d_shift": f32(c.B, width), "d_weight": f32(width), "d_post_weight": f32(width)}
        rcb.gated_norm_backward(c.cu, c.x, c.dy, torch.empty_like(c.x), branch=c.branch, dx_out=c.dx_out, **mods, **c.w, **c.kw, **got)
        runs.append(got)
    for n, t in runs[0].items():
        assert torch.isfinite(t).all(), n
        if t.dim() == 2:
            assert (t[empty] == 0).all(), n
        for other in runs[1:]:
            assert torch.equal(other[n], t), n
