"""The operators together, as the example uses them: a student's gradients against the same model in 32 bits on
plain torch operations, and a few training steps."""
import os
import sys

import pytest
import torch
import torch.nn.functional as F

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def plain_student(model, b, dim, axes, anchors):
    """The student's velocity in 32 bits, from the model's weights as fp32 leaves."""
    P = {n: p.detach().float().requires_grad_() for n, p in model.named_parameters()}
    freq = torch.cat([10000.0 ** (-2.0 * torch.arange(a // 2, device="cuda") / a) for a in axes])
    axis = torch.tensor([i for i, a in enumerate(axes) for _ in range(a // 2)], device="cuda")

    def rot(x, pos):
        ang = (pos.float()[:, axis] * freq)[:, None]
        u, v = x[..., 0::2], x[..., 1::2]
        return torch.stack((u * ang.cos() - v * ang.sin(), u * ang.sin() + v * ang.cos()), -1).flatten(-2)

    def rms(x, w):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w

    def attend(q, k, v):
        p = torch.softmax(torch.einsum("qhd,khd->hqk", q, k) * dim ** -0.5, -1)
        return torch.einsum("hqk,khd->qhd", p, v)

    per = lambda cu, t: torch.cat([t[i:i + 1].expand(y - x, -1) for i, (x, y) in enumerate(zip(cu, cu[1:]))])  # noqa: E731
    streams = [[b.cu_live, b.live.float(), b.pos_live, b.time.float(), None], [b.cu_static, b.static.float(), b.pos_static, b.time0.float(), None]]
    for i in range(len(model.blocks)):
        g = lambda n: P[f"blocks.{i}.{n}"]  # noqa: E731
        qkv = []
        for s in streams:
            cu, x, pos, time, add = s
            shift, scale, gate = F.linear(time, g("mod")).chunk(3, 1)
            s[1] = x = x if add is None else x + add
            y = F.layer_norm(x, x.shape[-1:], eps=1e-6) * (1 + per(cu, scale)) + per(cu, shift)
            q, k, v = F.linear(y, g("qkv")).view(len(x), 3, -1, dim).unbind(1)
            qkv.append((rot(rms(q, g("wq")), pos), rot(rms(k, g("wk")), pos), v))
            s[4] = per(cu, gate)
        live, static = [], []
        for r in range(len(b.cu_live) - 1):
            a, c = slice(b.cu_live[r], b.cu_live[r + 1]), slice(b.cu_static[r], b.cu_static[r + 1])
            ref = slice(c.start + anchors[r], c.stop)
            (ql, kl, vl), (qs, ks, vs) = qkv
            live.append(attend(ql[a], torch.cat((kl[a], ks[ref])), torch.cat((vl[a], vs[ref]))))
            static.append(attend(qs[c], ks[c], vs[c]))
        for s, o in zip(streams, (live, static)):
            s[4] = s[4] * F.linear(torch.cat(o).flatten(1), g("out"))
    x = streams[0][1] + streams[0][4]
    return F.linear(F.layer_norm(x, x.shape[-1:], eps=1e-6)[b.x_live], P["head"]), P


@pytest.mark.parametrize("heads, dim", [(4, 64), (2, 128)])
def test_student_gradients(heads, dim):
    import distill_block as ex

    reqs = ((16, 24, 12, 12, 2), (8, 40, 9, 13, 1), (0, 5, 7, 5, 1))
    axes = (dim // 8, 7 * dim // 16, 7 * dim // 16)
    model = ex.Model(2, heads, dim, seed=3).cuda()
    b = ex.Batch(reqs, heads * dim, seed=5)
    cache = ex.rc.RefCache(ex.rc.Segments(heads, dim, b.cu_live, b.cu_static, b.anchors, b.instr), num_layers=2)
    g = torch.randn(len(b.x_live), heads * dim, generator=torch.Generator().manual_seed(0)).cuda()
    v = ex.student_velocity(model, ex.rc.Rope(dim, axes=axes), b, cache)
    (v.float() * g).sum().backward()
    ref, P = plain_student(model, b, dim, axes, b.anchors)
    (ref * g).sum().backward()
    # Some 15 roundings to bf16 of relative size 2^-9 (rms) lie between a parameter and the loss, forwards and
    # backwards each, independent of one another: sqrt(30) 2^-9 = 1 %, and up to a few times that where a
    # norm or a softmax magnifies what comes in.
    rel = lambda a, r: ((a.float() - r).norm() / r.norm()).item()  # noqa: E731
    assert rel(v, ref) <= 0.04
    for n, p in model.named_parameters():
        assert rel(p.grad, P[n].grad) <= 0.06, n


def test_distillation_reduces_the_loss():
    import distill_block as ex

    losses, norms = ex.distil(steps=15)
    assert all(n > 0 for n in norms)
    assert losses[-1] < 0.7 * losses[0], losses
