"""The operators around the attention against their definitions in 64 bits:
one rounding to bf16 (unit roundoff U) of fp32 arithmetic (F relative to the
terms, a few dozen fp32 roundings)."""
import math

import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

pytestmark = pytest.mark.gpu

U, F = 2.0 ** -8, 2.0 ** -18
BF16 = torch.bfloat16


def gen_of(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rnd(g, *shape, gain=1.0, mean=0.0, dtype=BF16):
    return (torch.randn(*shape, generator=g, device="cuda") * gain + mean).to(dtype)


def check(name, got, ref, terms, rounding=U):
    """|got - ref| <= rounding |ref| + F terms, terms: the size of what was added up."""
    assert torch.isfinite(got).all(), name
    if got.numel():
        over = ((got.double() - ref).abs() - 1.01 * rounding * ref.abs() - F * terms - 1e-37).max().item()
        assert over <= 0, f"{name}: {over:.3e} above its bound"


# ---------------------------------------------------------------- qkv_rope
class RopeCase:
    def __init__(self, rows, H, D, axes, pairs, wdtype, out_rows=None, seed=0, span=40, theta=10000.0):
        g = gen_of(seed)
        self.H, self.D, self.axes, self.pairs, self.theta = H, D, axes, pairs, theta
        self.rope = rcb.Rope(D, axes, theta=theta, pairs=pairs)
        self.qkv = rnd(g, rows, 3, H, D, gain=1.5)
        self.w = [None, None] if wdtype is None else [rnd(g, D, gain=0.3, mean=1.0, dtype=wdtype) for _ in range(2)]
        self.pos = torch.randint(-span, span + 1, (rows, len(axes)), generator=g, device="cuda", dtype=torch.int32)
        self.out_rows = rows if out_rows is None else out_rows
        # rows scattered over the outputs; where these are fewer, some rows go nowhere
        perm = torch.randperm(max(rows, self.out_rows), generator=g, device="cuda")[:rows].to(torch.int32)
        if out_rows is not None and rows:
            perm[::7] = -1
        self.rows = perm if out_rows is not None else None
        self.kept = torch.ones(rows, dtype=torch.bool, device="cuda") if self.rows is None else (self.rows >= 0) & (self.rows < self.out_rows)
        self.to = torch.arange(rows, device="cuda") if self.rows is None else self.rows.long()
        self.grads = [rnd(g, self.out_rows, H, D) for _ in range(3)]

    def definition(self, x, w):
        if w is not None:
            x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
        ang = []
        for i, a in enumerate(self.axes):
            f = self.theta ** (-2.0 * torch.arange(a // 2, dtype=torch.float64, device="cuda") / max(a, 1))
            ang.append(self.pos[:, i:i + 1].double() * f)
        n = self.D // 2 - sum(self.axes) // 2
        ang = torch.cat(ang + [torch.zeros(len(x), n, dtype=torch.float64, device="cuda")], 1)[:, None]
        a, b = (x[..., 0::2], x[..., 1::2]) if self.pairs == "interleaved" else (x[..., :self.D // 2], x[..., self.D // 2:])
        u, v = a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()
        return torch.stack((u, v), -1).flatten(-2) if self.pairs == "interleaved" else torch.cat((u, v), -1)


ROPE = [
    (1, 1, 64, (64,), "interleaved", None, None),
    (1, 24, 128, (16, 56, 56), "halves", BF16, None),
    (37, 3, 128, (16, 56, 56), "interleaved", torch.float32, 53),
    (300, 5, 64, (8, 28, 28), "halves", torch.float32, 200),
    (65, 9, 128, (0, 40, 24), "interleaved", BF16, None),  # 64 dims not turned, an axis without dims
    (9, 2, 64, (2, 2, 2, 2), "halves", None, 4),
    (0, 2, 64, (8, 28, 28), "halves", None, 4),
    (5000, 2, 64, (8, 28, 28), "interleaved", BF16, None),
]


@pytest.mark.parametrize("case", ROPE, ids=lambda c: "-".join(str(x) for x in c[:3]))
def test_qkv_rope(case):
    c = RopeCase(*case)
    q, k, v = c.qkv.unbind(1)
    out = [torch.full((c.out_rows, c.H, c.D), 7.0, dtype=BF16, device="cuda") for _ in range(3)]
    rcb.qkv_rope(c.rope, c.pos, q, k, v, *out, *c.w, rows=c.rows)
    for i in range(3):
        x = c.qkv[:, i].double()
        w = c.w[i].double() if i < 2 and c.w[i] is not None else None
        ref = torch.full(out[i].shape, 7.0, dtype=torch.float64, device="cuda")
        ref[c.to[c.kept]] = (c.definition(x, w) if i < 2 else x)[c.kept]
        if i == 2:
            assert torch.equal(out[i].double(), ref)
        else:
            check("qk"[i], out[i], ref, ref.abs().amax(-1, keepdim=True) * 4 + 1)


@pytest.mark.parametrize("case", ROPE, ids=lambda c: "-".join(str(x) for x in c[:3]))
def test_qkv_rope_backward(case):
    c = RopeCase(*case)
    q, k, _ = c.qkv.unbind(1)
    dqkv = torch.full_like(c.qkv, float("nan"))
    dw = [None if w is None else torch.full((c.D,), float("nan"), device="cuda") for w in c.w]
    rcb.qkv_rope_backward(c.rope, c.pos, q, k, *c.grads, *dqkv.unbind(1), *c.w, *dw, rows=c.rows)
    g = [torch.zeros(c.qkv[:, 0].shape, dtype=torch.float64, device="cuda") for _ in range(3)]
    for i in range(3):
        g[i][c.kept] = c.grads[i][c.to[c.kept]].double()
    for i in range(2):
        x = c.qkv[:, i].double().requires_grad_()
        w = None if c.w[i] is None else c.w[i].double().requires_grad_()
        ref = torch.autograd.grad(c.definition(x, w), [x] if w is None else [x, w], g[i]) if len(x) else [x.detach(), torch.zeros(c.D, device="cuda").double()]
        size = g[i].abs().amax(-1, keepdim=True)
        if w is not None:  # the row's 1 / rms and the weight
            size = size * w.detach().abs().max() / (x.detach().square().mean(-1, keepdim=True) + 1e-6).sqrt()
        check("d" + "qk"[i], dqkv[:, i], ref[0], 16 * size)
        if w is not None:
            # each term g x / rms is a few fp32 roundings off; the sum of n of them loses at most n more, far fewer in parts
            xhat = (x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()).detach()
            terms = (g[i].abs().amax(-1, keepdim=True) * 2 * xhat.abs()).sum((0, 1))
            check("dw" + "qk"[i], dw[i], ref[1], terms, rounding=0)
    assert torch.equal(dqkv[:, 2].double(), g[2])


def test_rows_that_go_nowhere_may_hold_anything():
    """Padding: infinities and NaN in rows that the forward call drops reach neither their own gradient nor the weights'."""
    c = RopeCase(70, 3, 64, (8, 28, 28), "halves", BF16, 90, seed=3)
    lost = ~c.kept
    assert 0 < lost.sum() < 70
    dqkv, dw = [], []
    for fill in (1.0, math.nan, math.inf):
        x = c.qkv.clone()
        x[lost] = fill
        dqkv.append(torch.full_like(x, 7.0))
        dw.append([torch.empty(64, device="cuda") for _ in range(2)])
        rcb.qkv_rope_backward(c.rope, c.pos, x[:, 0], x[:, 1], *c.grads, *dqkv[-1].unbind(1), *c.w, *dw[-1], rows=c.rows)
    assert (dqkv[0][lost] == 0).all() and torch.isfinite(dw[0][0]).all()
    for i in (1, 2):
        assert torch.equal(dqkv[i], dqkv[0]) and all(torch.equal(a, b) for a, b in zip(dw[i], dw[0]))


def test_rope_angles_at_large_positions():
    """Position 2^24 at frequency 1: an fp32 product of the two would be right here, and off by a radian at the next pair."""
    c = RopeCase(50, 1, 64, (64,), "halves", None, span=2 ** 24)
    x = c.qkv[:, :1]
    out = torch.empty(50, 1, 64, dtype=BF16, device="cuda")
    rcb.qkv_rope(c.rope, c.pos, x[:, 0], None, None, out, None, None)
    ref = c.definition(x[:, 0].double(), None)
    check("q", out, ref, ref.abs().amax(-1, keepdim=True) * 4 + 1)


def test_rope_into_the_cache_slots():
    """K and V of the reference rows straight into a cache, then the in-slot build: as if packed first."""
    H, D, na, nr = 3, 128, 10, 150
    c = RopeCase(nr, H, D, (16, 56, 56), "interleaved", BF16, seed=4)
    seg = rcb.Segments(H, D, [0, 5], [0, na + nr], [na])
    a, b = rcb.RefCache(seg), rcb.RefCache(seg)
    q, k, v = c.qkv.unbind(1)
    packed = [torch.empty(nr, H, D, dtype=BF16, device="cuda") for _ in range(3)]
    rcb.qkv_rope(c.rope, c.pos, q, k, v, *packed, *c.w)
    rcb.qkv_rope(c.rope, c.pos, None, k, v, None, *a.kv(0), None, c.w[1])
    anchors = [rnd(gen_of(8), na, H, D) for _ in range(3)]
    st = [torch.cat((x, y)) for x, y in zip(anchors, packed)]
    o = [torch.empty_like(st[0]) for _ in range(2)]
    a.build_in_slot(0, st[0], anchors[1], anchors[2], o[0])
    for slot, t in zip(b.kv(0), packed[1:]):
        slot.copy_(t)
    b.build_in_slot(0, st[0], anchors[1], anchors[2], o[1])
    assert torch.equal(o[0], o[1]) and all(torch.equal(x, y) for x, y in zip(a.kv(0), b.kv(0)))


# ---------------------------------------------------------------- gated_norm
def norm64(t, kind):
    if kind == "layer":
        return (t - t.mean(-1, keepdim=True)) / (t.var(-1, unbiased=False, keepdim=True) + 1e-6).sqrt()
    return t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt() if kind == "rms" else t


class NormCase:
    def __init__(self, lens, width, norm, post, mdtype, weight, seed=0, mean=0.5):
        g = gen_of(seed)
        self.cu = [sum(lens[:i]) for i in range(len(lens) + 1)]
        n, B = self.cu[-1], len(lens)
        self.kw = {"norm": norm, "post_norm": post}
        self.x, self.branch, self.dy, self.dx_out = (rnd(g, n, width, gain=1.5, mean=m) for m in (mean, -0.3, 0.1, 0.0))
        mods = rnd(g, B, 3 * width + 16, gain=0.4, dtype=mdtype)
        self.mods = {m: mods[:, 8 + i * width:8 + (i + 1) * width] for i, m in enumerate(("gate", "scale", "shift"))}
        self.w = {"weight": rnd(g, width, gain=0.3, mean=1.0, dtype=mdtype) if weight else None,
                  "post_weight": rnd(g, width, gain=0.3, mean=1.0, dtype=mdtype) if weight and post else None}
        self.req = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(lens, device="cuda"))
        self.n, self.B, self.width = n, B, width


NORM = [
    ([1], 8, "layer", None, BF16, False),
    ([3, 0, 2], 64, "rms", "rms", torch.float32, True),
    ([5, 130, 1], 1000, "layer", "layer", BF16, True),
    ([33, 64], 2568, "rms", "layer", BF16, True),
    ([40, 0, 7], 4104, "layer", "rms", torch.float32, True),
    ([900], 256, None, "rms", BF16, False),
    ([17, 5], 8192, "layer", "rms", BF16, True),
    ([2] * 70 + [0, 9], 512, "rms", None, BF16, True),  # more requests than one launch takes
]
IDS = {"ids": lambda c: f"{len(c[0])}x{c[1]}-{c[2]}-{c[3]}"}


@pytest.mark.parametrize("case", NORM, **IDS)
def test_gated_norm(case):
    c = NormCase(*case)
    x_out, y = torch.empty_like(c.x), torch.full_like(c.x, float("nan"))
    rcb.gated_norm(c.cu, c.x, y, branch=c.branch, x_out=x_out, **c.mods, **c.w, **c.kw)
    one = torch.ones(c.width, dtype=torch.float64, device="cuda")
    w, pw = (one if t is None else t.double() for t in c.w.values())
    gate, scale, shift = (t.double()[c.req] for t in c.mods.values())
    t = c.x.double() + gate * (norm64(c.branch.double(), c.kw["post_norm"]) * pw)
    check("x_out", x_out, t, 16 * (c.x.double().abs() + gate.abs() * 6))
    that = norm64(t, c.kw["norm"])
    check("y", y, that * w * (1 + scale) + shift, 32 * ((1 + that.abs()) * (w * (1 + scale)).abs() + shift.abs() + t.abs().amax(-1, keepdim=True)))
    # without a branch, and in place
    y2 = torch.empty_like(y)
    rcb.gated_norm(c.cu, c.x, y2, scale=c.mods["scale"], shift=c.mods["shift"], weight=c.w["weight"], norm=c.kw["norm"])
    that = norm64(c.x.double(), c.kw["norm"])
    check("y of x", y2, that * w * (1 + scale) + shift, 32 * ((1 + that.abs()) * (w * (1 + scale)).abs() + shift.abs() + 8))
    x = c.x.clone()
    rcb.gated_norm(c.cu, x, None, branch=c.branch, x_out=x, gate=c.mods["gate"], post_weight=c.w["post_weight"], post_norm=c.kw["post_norm"], norm=None)
    assert torch.equal(x, x_out)


@pytest.mark.parametrize("case", NORM, **IDS)
def test_gated_norm_backward(case):
    c = NormCase(*case)
    f32 = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    got = {"dx": torch.empty_like(c.x), "d_branch": torch.empty_like(c.x), "d_gate": f32(c.B, c.width), "d_scale": f32(c.B, c.width),
           "d_shift": f32(c.B, c.width)}
    for n, t in c.w.items():
        if t is not None:
            got["d_" + n] = f32(c.width)
    mods = {n: c.mods[n] for n in ("gate", "scale")}
    rcb.gated_norm_backward(c.cu, c.x, c.dy, branch=c.branch, dx_out=c.dx_out, **mods, **c.w, **c.kw, **got)
    # the definition at x_out = c.x: the branch's part enters with value zero
    leaf = {"dx": c.x.double(), "d_branch": c.branch.double()}
    leaf.update({"d_" + n: t.double() for n, t in c.mods.items()})
    one = torch.ones(c.width, dtype=torch.float64, device="cuda")
    leaf.update({"d_" + n: one.clone() if t is None else t.double() for n, t in c.w.items()})
    leaf = {n: t.clone().requires_grad_() for n, t in leaf.items()}
    h = norm64(leaf["d_branch"], c.kw["post_norm"]) * leaf["d_post_weight"]
    add = leaf["d_gate"][c.req] * h
    t = leaf["dx"] + (add - add.detach())
    y = norm64(t, c.kw["norm"]) * leaf["d_weight"] * (1 + leaf["d_scale"][c.req]) + leaf["d_shift"][c.req]
    grads = dict(zip(leaf, torch.autograd.grad((y, t), list(leaf.values()), (c.dy.double(), c.dx_out.double()))))
    d = grads["dx"].abs().amax(-1, keepdim=True) + c.dy.double().abs().amax(-1, keepdim=True) * 8
    check("dx", got["dx"], grads["dx"], 32 * d)
    rb = 1.0 if c.kw["post_norm"] is None else 1 / (c.branch.double().square().mean(-1, keepdim=True)).sqrt().clamp_min(0.05)
    check("d_branch", got["d_branch"], grads["d_branch"], 64 * d * rb)
    which = torch.zeros(c.B, max(c.n, 1), dtype=torch.float64, device="cuda")
    if c.n:
        which[c.req, torch.arange(c.n, device="cuda")] = 1
    size = which[:, :c.n] @ (d.expand(c.n, c.width) * 8)  # what a request's rows add up, column by column
    for n in ("d_gate", "d_scale", "d_shift"):
        check(n, got[n], grads[n], 16 * size, rounding=0)
    for n in ("d_weight", "d_post_weight"):
        if n in got:
            check(n, got[n], grads[n], 32 * size.sum(0), rounding=0)
    again = {n: torch.empty_like(t) for n, t in got.items()}
    rcb.gated_norm_backward(c.cu, c.x, c.dy, branch=c.branch, dx_out=c.dx_out, **mods, **c.w, **c.kw, **again)
    assert all(torch.equal(a, b) for a, b in zip(got.values(), again.values()))


@pytest.mark.parametrize("case", [
    ([70, 0, 95], 200, "rms", None, BF16, False),  # many blocks a request, each request by itself
    ([3] * 40, 136, "layer", "rms", torch.float32, False),  # few
    ([9] * 40, 136, "layer", None, torch.float32, True),  # few, added up over the requests
    ([1500, 1, 900], 2056, "rms", "rms", BF16, True),  # blocks that take several rows and go on to the next request
    ([1100, 1300], 1032, "layer", "layer", BF16, False),
], **IDS)
def test_gated_norm_backward_sums(case):
    """The forms in which the parameters' gradients are added up."""
    test_gated_norm_backward(case)


def test_gated_norm_backward_of_parts():
    """Only the norm (no branch), and only the residual (no y)."""
    c = NormCase([30, 12], 512, "layer", None, BF16, False)
    dx, ds = torch.empty_like(c.x), torch.empty(2, 512, device="cuda")
    rcb.gated_norm_backward(c.cu, c.x, c.dy, dx, scale=c.mods["scale"], d_shift=ds)
    x = c.x.double().requires_grad_()
    y = norm64(x, "layer") * (1 + c.mods["scale"].double()[c.req])
    (ref,) = torch.autograd.grad(y, x, c.dy.double())
    check("dx", dx, ref, 32 * c.dy.double().abs().amax(-1, keepdim=True) * 4)
    ref = torch.stack([c.dy[:30].double().sum(0), c.dy[30:].double().sum(0)])
    check("d_shift", ds, ref, 30 * 6, rounding=0)
    db, dg = torch.empty_like(c.x), torch.empty(2, 512, device="cuda")
    rcb.gated_norm_backward(c.cu, None, None, dx, branch=c.branch, dx_out=c.dx_out, gate=c.mods["gate"], d_branch=db, d_gate=dg, norm=None)
    assert torch.equal(dx, c.dx_out)
    check("d_branch", db, c.dx_out.double() * c.mods["gate"].double()[c.req], 4)
    prod = c.dx_out.double() * c.branch.double()
    check("d_gate", dg, torch.stack([prod[:30].sum(0), prod[30:].sum(0)]), 30 * 30, rounding=0)


def test_one_modulation_for_all_requests():
    """An expanded row of scale and shift is read as the same rows apart."""
    c = NormCase([5, 0, 7], 512, "rms", None, BF16, False)
    one = {k: t[:1] for k, t in c.mods.items()}
    want, got = torch.empty_like(c.x), torch.empty_like(c.x)
    rcb.gated_norm(c.cu, c.x, want, branch=c.branch, norm="rms", **{k: t.repeat(3, 1) for k, t in one.items()})
    rcb.gated_norm(c.cu, c.x, got, branch=c.branch, norm="rms", **{k: t.expand(3, -1) for k, t in one.items()})
    assert torch.equal(want, got)


def test_calls_replay_from_a_cuda_graph():
    r = RopeCase(70, 3, 128, (16, 56, 56), "halves", BF16, out_rows=80)
    n = NormCase([30, 12], 4096, "layer", "rms", BF16, True)  # (rows ahead of more shared memory than a launch has by default)
    g = tensors([300, 5000], (BF16,), 1.0)
    out = [torch.zeros(80, 3, 128, dtype=BF16, device="cuda") for _ in range(3)]
    dqkv, dw = torch.zeros_like(r.qkv), [torch.zeros(128, device="cuda") for _ in range(2)]
    y, dx, dg, clipped = torch.zeros_like(n.x), torch.zeros_like(n.x), torch.zeros(2, 4096, device="cuda"), [torch.zeros_like(t) for t in g]
    norm = torch.zeros((), device="cuda")

    def calls():
        q, k, v = r.qkv.unbind(1)
        rcb.qkv_rope(r.rope, r.pos, q, k, v, *out, *r.w, rows=r.rows)
        rcb.qkv_rope_backward(r.rope, r.pos, q, k, *r.grads, *dqkv.unbind(1), *r.w, *dw, rows=r.rows)
        rcb.gated_norm(n.cu, n.x, y, branch=n.branch, **n.mods, **n.w, **n.kw)
        rcb.gated_norm_backward(n.cu, n.x, n.dy, dx, branch=n.branch, gate=n.mods["gate"], d_gate=dg, **n.w, **n.kw)
        rcb.clip_gradients(g, 0.5, out=clipped, norm=norm)

    results = [*out, dqkv, *dw, y, dx, dg, *clipped, norm]
    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in results]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for t in results:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(results, want))


def test_norm_of_a_large_mean():
    """Mean 1000, deviation 4 (the spacing of bf16 there): squares would cancel, deviations do not."""
    g = gen_of(2)
    x = rnd(g, 20, 4096, gain=4.0, mean=1000.0)
    y = torch.empty_like(x)
    rcb.gated_norm([0, 20], x, y)
    ref = norm64(x.double(), "layer")
    # the mean is 1000 to 2^-23 of itself: 2^-13 of a deviation
    check("y", y, ref, 1000 / 4 * torch.ones_like(ref))


# ---------------------------------------------------------------- clip_gradients
def tensors(sizes, dtypes, gain, seed=0, odd=False):
    g = gen_of(seed)
    out = []
    for i, n in enumerate(sizes):
        dt = dtypes[i % len(dtypes)]
        buf = rnd(g, n + 8, gain=gain, dtype=dt)
        out.append(buf[1 + i % 7:1 + i % 7 + n] if odd else buf[:n])
    return out


@pytest.mark.parametrize("sizes", [[1], [0, 5, 0], [3, 17, 16384, 16385, 40000], list(range(1, 600)), [3_000_001]], ids=len)
@pytest.mark.parametrize("dtypes", [(BF16,), (torch.float32,), (BF16, torch.float32)], ids=["bf16", "fp32", "both"])
@pytest.mark.parametrize("odd", [False, True])
def test_clip_gradients(sizes, dtypes, odd):
    for gain, out32 in ((1.0, False), (1e-9, True), (1.0, True)):
        grads = tensors(sizes, dtypes, gain, odd=odd)
        before = [t.clone() for t in grads]
        norm64 = math.sqrt(sum(t.double().square().sum().item() for t in grads))
        coef = min(1.0, 0.05 / (norm64 + 1e-6))
        outs = [torch.full((t.numel() + 9,), 7.0, dtype=torch.float32 if out32 else t.dtype, device="cuda")[1:1 + t.numel()] for t in grads]
        norm = rcb.clip_gradients(grads, 0.05, out=outs)
        assert abs(norm.item() - norm64) <= 1e-5 * norm64
        for g, o, b in zip(grads, outs, before):
            assert torch.equal(g, b)
            check("out", o, g.double() * coef, g.double().abs() * coef * 4, rounding=U if o.dtype is BF16 else 0)
            assert o._base[0] == 7.0 and (o._base[1 + o.numel():] == 7.0).all()  # nothing beside it
        again = rcb.clip_gradients(grads, 0.05)
        assert torch.equal(again, norm)
        for g, o in zip(grads, outs):
            if not out32 or o.dtype is g.dtype:
                assert torch.equal(g, o)


def test_clip_of_special_values():
    g = tensors([100, 200], (BF16, torch.float32), 1.0)
    assert rcb.clip_gradients(g, math.inf).item() > 1
    keep = [t.clone() for t in g]
    rcb.clip_gradients(g, 1e9)
    assert all(torch.equal(a, b) for a, b in zip(g, keep))
    rcb.clip_gradients(g, 0.0)
    assert all((t == 0).all() for t in g)
    g[0][3] = math.inf
    g[1].fill_(2.0)
    assert rcb.clip_gradients(g, 1.0).item() == math.inf
    assert (g[1] == 0).all() and g[0][3].isnan()
    g[1][0] = math.nan
    assert math.isnan(rcb.clip_gradients(g, 1.0).item())
    assert all(t.isnan().all() for t in g)
    assert rcb.clip_gradients([], 1.0).item() == 0.0


def test_largest_finite_bound_is_a_bound():
    g = torch.tensor([math.inf, 2.0], device="cuda")
    assert rcb.clip_gradients([g], 3.3e38).item() == math.inf
    assert g[0].isnan() and g[1] == 0


def test_other_stream():
    c = NormCase([30, 12], 512, "layer", "rms", BF16, True)
    side = torch.cuda.Stream()
    want, got = torch.empty_like(c.x), torch.zeros_like(c.x)
    a, b = (torch.empty(2, 512, device="cuda") for _ in range(2))
    kw = dict(branch=c.branch, dx_out=c.dx_out, gate=c.mods["gate"], scale=c.mods["scale"], **c.w, **c.kw)
    rcb.gated_norm_backward(c.cu, c.x, c.dy, want, d_gate=a, **kw)
    torch.cuda.synchronize()
    rcb.gated_norm_backward(c.cu, c.x, c.dy, got, d_gate=b, stream=side, **kw)
    side.synchronize()
    assert torch.equal(want, got) and torch.equal(a, b)


@pytest.mark.parametrize("handle", [False, True])
def test_memory_for_another_stream_is_that_streams(handle):
    """A block that the current stream has just freed may still be in use there: a call on another stream must not get it."""
    side = torch.cuda.Stream()
    g = torch.ones(1000, device="cuda")
    rcb.clip_gradients([g], math.inf)
    torch.cuda.synchronize()
    on = side.cuda_stream if handle else side
    for nbytes in (512, 3 << 20):
        x = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        freed = x.data_ptr()
        del x
        assert rcb._work(nbytes, g, on).data_ptr() != freed
        x = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        assert x.data_ptr() == freed  # (it was there to be had)
        del x
    x = torch.empty((), device="cuda")
    freed = x.data_ptr()
    del x
    norm = rcb.clip_gradients([g], math.inf, stream=on)
    assert norm.data_ptr() != freed
    side.synchronize()
    assert abs(norm.item() - 1000 ** 0.5) < 1e-4


def test_refusals_of_tensors():
    c = RopeCase(6, 2, 64, (8, 28, 28), "halves", BF16)
    q, k, v = c.qkv.unbind(1)
    out = [torch.empty(6, 2, 64, dtype=BF16, device="cuda") for _ in range(3)]
    with pytest.raises(ValueError, match="positions"):
        rcb.qkv_rope(c.rope, c.pos.long(), q, k, v, *out)
    with pytest.raises(ValueError, match="bf16"):
        rcb.qkv_rope(c.rope, c.pos, q.float(), k, v, *out)
    with pytest.raises(ValueError, match="contiguous"):
        rcb.qkv_rope(c.rope, c.pos, torch.empty(2, 6, 64, dtype=BF16, device="cuda").transpose(0, 1), k, v, *out)
    with pytest.raises(ValueError, match="one type"):
        rcb.qkv_rope(c.rope, c.pos, q, k, v, *out, c.w[0], c.w[1].float())
    with pytest.raises(rcb.RefCacheError, match="without its output"):
        rcb.qkv_rope(c.rope, c.pos, q, k, v, out[0], out[1], None)
    with pytest.raises(rcb.RefCacheError, match="do not fit"):
        rcb.qkv_rope(c.rope, c.pos, q, k, v, *(t[:5] for t in out))
    n = NormCase([4], 64, "layer", None, BF16, False)
    y = torch.empty_like(n.x)
    with pytest.raises(ValueError, match="scale"):
        rcb.gated_norm([0, 2, 4], n.x, y, scale=n.mods["scale"])
    with pytest.raises(rcb.RefCacheError, match="aligned"):
        rcb.gated_norm(n.cu, n.x, y, weight=torch.zeros(65, dtype=BF16, device="cuda")[1:])
    with pytest.raises(rcb.RefCacheError, match="without a branch"):
        rcb.gated_norm(n.cu, n.x, y, x_out=torch.empty_like(y))
    with pytest.raises(ValueError, match="elements"):
        rcb.clip_gradients([n.x], 1.0, out=[n.x[:2]])
    with pytest.raises(ValueError, match="bf16 or float32"):
        rcb.clip_gradients([n.x.half()], 1.0)
