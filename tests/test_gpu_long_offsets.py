"""The gradients and the operators around the attention on tensors of more than 2^31 elements: the last rows must be
what a call on these rows alone gives."""
import math

import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
GB = 1 << 30


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.mem_get_info()[0] < 70 * GB:
        pytest.skip("needs 70 GB of device memory")
    yield
    torch.cuda.empty_cache()
    assert rcb.status() == rcb.OK, rcb.last_error()


def rnd(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda", dtype=BF16)


def step_gradients(n, x):
    """Gradients of a step of n requests of 256 live and 256 cached rows; x stands for all inputs."""
    H, D = x.shape[1:]
    seg = rcb.Segments(H, D, [256 * i for i in range(n + 1)], [256 * i for i in range(n + 1)], [0] * n, [0] * n)
    cache = rcb.RefCache(seg)
    out = {m: torch.empty_like(x) for m in ("dq", "dk", "dv", "dk_ref", "dv_ref")}
    cache.build(0, x, x, x, out["dq"])
    lse = torch.full(x.shape[:2], 16.0, device="cuda")  # above every score: weights below 1
    cache.step_backward(0, x, x, x, x, lse, x, **out)
    torch.cuda.synchronize()
    cache.close()
    return out


@pytest.mark.parametrize("H, D", [(64, 128), (64, 64)])
def test_attention_gradients(H, D):
    n = (1 << 31) // (256 * H * D) + 5
    x = rnd(0, 256 * n, H, D)
    assert x.numel() > 1 << 31
    long = step_gradients(n, x)
    tail = x[-256:].clone()
    alone = step_gradients(1, tail)
    for m, t in alone.items():
        assert torch.isfinite(t).all() and t.abs().max() > 0, m
        assert torch.equal(long[m][-256:], t), m


def test_qkv_rope():
    H, D, rows, last = 64, 128, 90_000, 100
    rope = rcb.Rope(D, (16, 56, 56))
    qkv, w = rnd(1, rows, 3, H, D), [rnd(2, D), rnd(3, D)]
    assert qkv.numel() > 1 << 31
    pos = torch.arange(3 * rows, device="cuda", dtype=torch.int32).reshape(rows, 3) % 977
    out = [torch.empty(rows, H, D, dtype=BF16, device="cuda") for _ in range(3)]
    rcb.qkv_rope(rope, pos, *qkv.unbind(1), *out, *w)
    d = torch.empty_like(qkv)
    rcb.qkv_rope_backward(rope, pos, qkv[:, 0], qkv[:, 1], *out, *d.unbind(1), *w)
    some, p = qkv[-last:].clone(), pos[-last:].clone()
    want = [torch.empty(last, H, D, dtype=BF16, device="cuda") for _ in range(3)]
    rcb.qkv_rope(rope, p, *some.unbind(1), *want, *w)
    dwant = torch.empty_like(some)
    rcb.qkv_rope_backward(rope, p, some[:, 0], some[:, 1], *want, *dwant.unbind(1), *w)
    assert all(torch.equal(a[-last:], b) for a, b in zip(out, want))
    assert torch.equal(d[-last:], dwant)


def test_gated_norm():
    width, rows, last = 8192, 270_000, 50
    cu = [0, rows - last, rows]
    x, branch = rnd(4, rows, width), rnd(5, rows, width)
    assert x.numel() > 1 << 31
    gate, scale, shift = (rnd(6 + i, 2, width) for i in range(3))
    y, x_out = torch.empty_like(x), torch.empty_like(x)
    rcb.gated_norm(cu, x, y, branch=branch, x_out=x_out, gate=gate, scale=scale, shift=shift, post_norm="rms")
    xs, bs, m = x[-last:].clone(), branch[-last:].clone(), dict(gate=gate[1:].clone(), scale=scale[1:].clone())
    ys, xo = torch.empty_like(xs), torch.empty_like(xs)
    rcb.gated_norm([0, last], xs, ys, branch=bs, x_out=xo, shift=shift[1:].clone(), post_norm="rms", **m)
    assert torch.equal(y[-last:], ys) and torch.equal(x_out[-last:], xo)
    dx, db = y, x  # (written over what is not needed any more)
    rcb.gated_norm_backward(cu, x_out, branch, dx, branch=branch, d_branch=db, gate=gate, scale=scale, post_norm="rms")
    dxs, dbs = torch.empty_like(xs), torch.empty_like(xs)
    rcb.gated_norm_backward([0, last], xo, bs, dxs, branch=bs, d_branch=dbs, post_norm="rms", **m)
    assert torch.equal(dx[-last:], dxs) and torch.equal(db[-last:], dbs)


def test_clip_gradients():
    g = [torch.ones((1 << 31) + 100_003, dtype=BF16, device="cuda"), torch.full((7,), 2.0, device="cuda")]
    norm = math.sqrt(g[0].numel() + 28)
    assert abs(rcb.clip_gradients(g, 100.0).item() / norm - 1) < 1e-6
    want = torch.tensor(100.0 / norm, dtype=torch.float64)
    assert (g[0] == want.to(BF16)).all()
    assert (g[1].double() / (2 * want) - 1).abs().max() < 1e-6
