"""Teacher-forced distillation of a small student through the beyond mask, on this library's operators.

The teacher attends all of [LT; X_t; R] at every step (full attention); the student computes its reference rows once,
beside their static anchors, and its live rows over the reference cache.  Both are a few transformer blocks with the
same weights at first; the student is trained on the squared distance of the two velocities on the target rows, as in
the paper's first stage.  A block is: gated residual and modulated norm, projection, per-head norms and rotary
positions, joint attention, output projection; the library runs all of it but the projections (torch) forwards and
backwards, and clips the gradients.

    python examples/distill_block.py [--steps 30]

It also shows how the calls are tied into torch's autograd: one Function for each call, the cached rows' keys and
values as outputs of the prefill and inputs of the step, so that several steps that share a cache add their gradients up.
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_21229_gb300 import refcache as rc  # noqa: E402

BF16 = torch.bfloat16


# ---------------------------------------------------------------- the library's calls as autograd functions
class GatedNorm(torch.autograd.Function):
    """(x + gate * branch, its norm modulated by scale and shift); branch and gate may be None."""

    @staticmethod
    def forward(ctx, cu, x, branch, gate, scale, shift):
        y = torch.empty_like(x)
        x_out = x if branch is None else torch.empty_like(x)
        rc.gated_norm(cu, x, y, branch=branch, x_out=None if branch is None else x_out, gate=gate, scale=scale, shift=shift)
        ctx.cu = cu
        ctx.save_for_backward(x_out, branch, gate, scale)
        return x_out, y

    @staticmethod
    def backward(ctx, dx_out, dy):
        x_out, branch, gate, scale = ctx.saved_tensors
        f32 = lambda t: torch.empty(scale.shape, dtype=torch.float32, device=dy.device)  # noqa: E731
        dx, d_scale, d_shift = torch.empty_like(x_out), f32(scale), f32(scale)
        d_branch, d_gate = (None, None) if branch is None else (torch.empty_like(branch), f32(gate))
        rc.gated_norm_backward(ctx.cu, x_out, dy.contiguous(), dx, branch=branch, dx_out=dx_out.contiguous(), d_branch=d_branch, gate=gate,
                               scale=scale, d_gate=d_gate, d_scale=d_scale, d_shift=d_shift)
        to = lambda t: None if t is None else t.to(scale.dtype)  # noqa: E731
        return None, dx, d_branch, to(d_gate), to(d_scale), to(d_shift)


class QkvRope(torch.autograd.Function):
    """q, k and v of the attention from a fused projection [rows, 3, H, D]."""

    @staticmethod
    def forward(ctx, rope, positions, qkv, wq, wk):
        q, k, v = qkv.unbind(1)
        out = [torch.empty(q.shape, dtype=BF16, device=qkv.device) for _ in range(3)]
        rc.qkv_rope(rope, positions, q, k, v, *out, wq, wk)
        ctx.rope = rope
        ctx.save_for_backward(positions, qkv, wq, wk)
        return tuple(out)

    @staticmethod
    def backward(ctx, dq, dk, dv):
        positions, qkv, wq, wk = ctx.saved_tensors
        q, k, _ = qkv.unbind(1)
        dqkv = torch.empty_like(qkv)
        dwq, dwk = (torch.empty(wq.shape, dtype=torch.float32, device=qkv.device) for _ in range(2))
        rc.qkv_rope_backward(ctx.rope, positions, q, k, dq.contiguous(), dk.contiguous(), dv.contiguous(), *dqkv.unbind(1), wq, wk, dwq, dwk)
        return None, None, dqkv, dwq.to(wq.dtype), dwk.to(wk.dtype)


class Prefill(torch.autograd.Function):
    """The static rows' attention, and the cached rows' keys and values."""

    @staticmethod
    def forward(ctx, cache, layer, q, k, v):
        o = torch.empty_like(q)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        cache.build(layer, q, k, v, o, lse)
        ctx.cache, ctx.layer = cache, layer
        ctx.save_for_backward(q, k, v, o, lse)
        return (o, *cache.kv(layer))

    @staticmethod
    def backward(ctx, d_o, dk_ref, dv_ref):
        q, k, v, o, lse = ctx.saved_tensors
        dq, dk, dv = (torch.empty_like(q) for _ in range(3))
        ctx.cache.build_backward(ctx.layer, q, k, v, o, lse, d_o.contiguous(), dq, dk, dv, dk_ref.contiguous(), dv_ref.contiguous())
        return None, None, dq, dk, dv


class Step(torch.autograd.Function):
    """The live rows' attention over their own keys and the cache's."""

    @staticmethod
    def forward(ctx, cache, layer, q, k, v, k_ref, v_ref):
        o = torch.empty_like(q)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        cache.step(layer, q, k, v, o, lse)
        ctx.cache, ctx.layer = cache, layer
        ctx.save_for_backward(q, k, v, o, lse)
        return o

    @staticmethod
    def backward(ctx, d_o):
        q, k, v, o, lse = ctx.saved_tensors
        dq, dk, dv = (torch.empty_like(q) for _ in range(3))
        dk_ref, dv_ref = (torch.empty_like(t) for t in ctx.cache.kv(ctx.layer))
        ctx.cache.step_backward(ctx.layer, q, k, v, o, lse, d_o.contiguous(), dq, dk, dv, dk_ref, dv_ref)
        return None, None, dq, dk, dv, dk_ref, dv_ref


# ---------------------------------------------------------------- the model
class Block(torch.nn.Module):
    def __init__(self, heads, dim, gen):
        super().__init__()
        c = heads * dim
        w = lambda *s, std: torch.nn.Parameter((torch.randn(*s, generator=gen) * std).to(BF16))  # noqa: E731
        self.heads, self.dim = heads, dim
        self.qkv, self.out = w(3 * c, c, std=c ** -0.5), w(c, c, std=c ** -0.5)
        self.mod = w(3 * c, c, std=0.3 * c ** -0.5)  # shift, scale and gate from a request's time embedding
        self.wq, self.wk = (torch.nn.Parameter(torch.ones(dim, dtype=BF16)) for _ in range(2))

    def project(self, y, rope, positions):
        return QkvRope.apply(rope, positions, F.linear(y, self.qkv).view(-1, 3, self.heads, self.dim), self.wq, self.wk)

    def merge(self, o):
        return F.linear(o.flatten(1), self.out)

    def modulation(self, time):
        return F.linear(time, self.mod).chunk(3, 1)


class Model(torch.nn.Module):
    def __init__(self, layers, heads, dim, seed=0):
        super().__init__()
        gen = torch.Generator().manual_seed(seed)
        self.blocks = torch.nn.ModuleList(Block(heads, dim, gen) for _ in range(layers))
        c = heads * dim
        self.head = torch.nn.Parameter((torch.randn(c, c, generator=gen) * c ** -0.5).to(BF16))


class Stream:
    """Rows that go through the blocks: x, with the branch and gate of the half before still to be added."""

    def __init__(self, cu, x, positions, time):
        self.cu, self.x, self.positions, self.time, self.branch, self.gate = cu, x, positions, time, None, None

    def enter(self, block):
        shift, scale, gate = block.modulation(self.time)
        self.x, y = GatedNorm.apply(self.cu, self.x, self.branch, self.gate, scale, shift)
        self.gate = gate
        return y

    def leave(self):
        zero = torch.zeros_like(self.gate)
        return GatedNorm.apply(self.cu, self.x, self.branch, self.gate, zero, zero)[1]


class Batch:
    """Requests of (anchor, instruction, target height x width, references) tokens with random contents."""

    def __init__(self, reqs, c, seed):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        rnd = lambda n: torch.randn(n, c, generator=gen, device="cuda").to(BF16)  # noqa: E731
        self.cu_live, self.cu_static, self.cu_full = [0], [0], [0]
        live, static, full, pl, ps, pf, target = [], [], [], [], [], [], []
        for n_st, n_lt, h, w, refs in reqs:
            text = torch.arange(max(n_st, n_lt), device="cuda", dtype=torch.int32)[:, None].expand(-1, 3) + max(h, w)
            grid = torch.stack(torch.meshgrid(torch.arange(refs + 1), torch.arange(h) - h // 2, torch.arange(w) - w // 2, indexing="ij"), -1)
            grid = grid.reshape(-1, 3).int().cuda()
            lt, x, st, r = rnd(n_lt), rnd(h * w), rnd(n_st), rnd(refs * h * w)
            live += [lt, x]
            static += [st, r]
            full += [lt, x, r]
            pl += [text[:n_lt], grid[:h * w]]
            ps += [text[:n_st], grid[h * w:]]
            pf += [text[:n_lt], grid]
            target.append((self.cu_live[-1] + n_lt, self.cu_full[-1] + n_lt, h * w))
            self.cu_live.append(self.cu_live[-1] + n_lt + h * w)
            self.cu_static.append(self.cu_static[-1] + n_st + refs * h * w)
            self.cu_full.append(self.cu_full[-1] + n_lt + (refs + 1) * h * w)
        self.live, self.static, self.full = (torch.cat(t) for t in (live, static, full))
        self.pos_live, self.pos_static, self.pos_full = (torch.cat(t).contiguous() for t in (pl, ps, pf))
        rows = lambda i: torch.cat([torch.arange(t[i], t[i] + t[2], device="cuda") for t in target])  # noqa: E731
        self.x_live, self.x_full = rows(0), rows(1)
        self.time, self.time0 = rnd(len(reqs)), rnd(1).expand(len(reqs), c).contiguous()
        self.anchors, self.instr = [r[0] for r in reqs], [r[1] for r in reqs]


def teacher_velocity(model, rope, b):
    s = Stream(b.cu_full, b.full, b.pos_full, b.time)
    for block in model.blocks:
        q, k, v = block.project(s.enter(block), rope, s.positions)
        o = torch.empty_like(q)
        rc.full_attention(b.cu_full, q, k, v, o)
        s.branch = block.merge(o)
    return F.linear(s.leave()[b.x_full], model.head)


def student_velocity(model, rope, b, cache):
    live, static = Stream(b.cu_live, b.live, b.pos_live, b.time), Stream(b.cu_static, b.static, b.pos_static, b.time0)
    for layer, block in enumerate(model.blocks):
        o, k_ref, v_ref = Prefill.apply(cache, layer, *block.project(static.enter(block), rope, static.positions))
        static.branch = block.merge(o)
        live.branch = block.merge(Step.apply(cache, layer, *block.project(live.enter(block), rope, live.positions), k_ref, v_ref))
    return F.linear(live.leave()[b.x_live], model.head)


def distil(steps=30, layers=2, heads=4, dim=64, reqs=((16, 24, 12, 12, 2), (8, 40, 9, 13, 1)), lr=2e-4, max_norm=0.05):
    """The losses of `steps` steps on one batch, and the gradients' norms before clipping."""
    rope = rc.Rope(dim, axes=(dim // 8, 7 * dim // 16, 7 * dim // 16))
    teacher, student = (Model(layers, heads, dim).cuda() for _ in range(2))
    b = Batch(reqs, heads * dim, seed=1)
    cache = rc.RefCache(rc.Segments(heads, dim, b.cu_live, b.cu_static, b.anchors, b.instr), num_layers=layers)
    with torch.no_grad():
        goal = teacher_velocity(teacher, rope, b).float()
    params = list(student.parameters())
    opt = torch.optim.AdamW(params, lr=lr)
    losses, norms = [], []
    for _ in range(steps):
        opt.zero_grad(set_to_none=True)
        loss = (student_velocity(student, rope, b, cache).float() - goal).square().mean()
        loss.backward()
        norms.append(rc.clip_gradients([p.grad for p in params if p.grad is not None], max_norm))
        opt.step()
        losses.append(loss.detach())
    if rc.status() != rc.OK:
        raise RuntimeError(rc.last_error())
    return [float(x) for x in losses], [float(x) for x in norms]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    for i, (loss, norm) in enumerate(zip(*distil(ap.parse_args().steps))):
        print(f"step {i:3d}  loss {loss:.5f}  gradient norm {norm:.4f}")
