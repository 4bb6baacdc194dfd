"""Gradients of the attention calls against the same in 64 bits, element by
element, within bounds that follow from the roundings the calls promise: P and
dS to bf16 as operands, O (an input, from which the row sums dO . O are taken)
and the gradients themselves to bf16, everything else fp32."""
import math

import pytest
import torch

import workloads
from paper_2608_21229_gb300 import refcache as rcb

pytestmark = pytest.mark.gpu

U = 2.0 ** -8  # unit roundoff of bf16
F = 2.0 ** -15  # allowance for fp32 scores (|s| < 2^6 to 2^-21 of it), ex2 and sums, relative to the terms
KERNELS = ["tcgen05", "mma_sync"]


@pytest.fixture(autouse=True)
def default_kernel():
    old = rcb.set_kernel("tcgen05")
    yield
    rcb.set_kernel(old)
    assert rcb.status() == rcb.OK, rcb.last_error()


def rnd(gen, *shape, gain=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * gain).to(torch.bfloat16)


class Ref:
    """Sums of the gradients, and of their bounds, over groups of rows that see the same keys."""

    def __init__(self, forward=False):
        """forward: o and lse come from the library's forward call, whose P is rounded to bf16 before P V and whose
        lse is within 2e-3 (the bound of its own tests)."""
        self.sums, self.forward, self.lse_abs = {}, forward, 2e-3 if forward else 0.0

    def add(self, name, rows, shape, val, bound):
        if name not in self.sums:
            self.sums[name] = [torch.zeros(shape, dtype=torch.float64, device="cuda") for _ in range(2)]
        for t, x in zip(self.sums[name], (val, bound)):
            t[rows] += x.transpose(0, 1)

    def group(self, q, do, keys, scale, dq, o=None):
        """q, do [n, H, D] of one group; keys: (K, V, (name, rows, shape) of dK or None, of dV); dq: where dQ goes.
        Returns the exact o and log-sum-exp."""
        hf = lambda t: t.double().transpose(0, 1)  # noqa: E731
        K, V = hf(torch.cat([k[0] for k in keys])), hf(torch.cat([k[1] for k in keys]))
        q, do = hf(q), hf(do)
        s = q @ K.transpose(1, 2) * scale
        lse = torch.logsumexp(s, -1)
        p = torch.exp(s - lse[..., None])
        out = p @ V
        dp = do @ V.transpose(1, 2)
        delta = (p * dp).sum(-1, keepdim=True)
        ds = p * (dp - delta)
        # |error| of each dS: its own rounding, the row sum's (O rounded), P's through lse, exp and scores
        rel = F + self.lse_abs
        eds = U * ds.abs() + p * ((U + F) * (do.abs() * out.abs()).sum(-1, keepdim=True) + F * (do.abs() @ V.abs().transpose(1, 2)))
        if self.forward:
            eds = eds + p * U * (do.abs() * (p @ V.abs())).sum(-1, keepdim=True)
        eds = eds + rel * ds.abs()
        ep = (U + rel) * p
        add = lambda where, val, err: where and self.add(*where, val, err + U * val.abs())  # noqa: E731
        add(dq, scale * ds @ K, scale * eds @ K.abs())
        dk, dv = scale * ds.transpose(1, 2) @ q, p.transpose(1, 2) @ do
        ek, ev = scale * eds.transpose(1, 2) @ q.abs(), ep.transpose(1, 2) @ do.abs()
        at = 0
        for k in keys:
            n = slice(at, at + len(k[0]))
            at += len(k[0])
            add(k[2], dk[:, n], ek[:, n])
            add(k[3], dv[:, n], ev[:, n])
        return out.transpose(0, 1), lse.transpose(0, 1)

    def check(self, name, got, extra=None):
        ref, bound = self.sums.get(name, (torch.zeros(got.shape, dtype=torch.float64, device="cuda"),) * 2)
        if extra is not None:  # added before the rounding
            ref = ref + extra.double()
            bound = bound + U * ref.abs()
        assert torch.isfinite(got).all(), f"{name}: not finite"
        over = ((got.double() - ref).abs() - 1.01 * bound - 1e-30).max().item() if got.numel() else 0.0
        assert over <= 0, f"{name}: {over:.3e} above its bound (largest bound {bound.max().item():.3e})"


class Case:
    def __init__(self, heads, dim, reqs, mask="beyond", seed=0, gain=1.0):
        self.H, self.D, self.reqs, self.mask = heads, dim, reqs, mask
        cu = lambda lens: [sum(lens[:i]) for i in range(len(lens) + 1)]  # noqa: E731
        self.cu_live, self.cu_static = cu([r[1] + r[2] for r in reqs]), cu([r[0] + r[3] for r in reqs])
        self.seg = rcb.Segments(heads, dim, self.cu_live, self.cu_static, [r[0] for r in reqs], [r[1] for r in reqs])
        self.cache = rcb.RefCache(self.seg, mask_mode=mask)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        shape = lambda n: (n, heads, dim)  # noqa: E731
        self.live = [rnd(gen, *shape(self.cu_live[-1]), gain=g) for g in (gain, 1, 1, 1)]  # q, k, v, do
        self.static = [rnd(gen, *shape(self.cu_static[-1]), gain=g) for g in (gain, 1, 1, 1)]
        rows = []
        for b, r in enumerate(reqs):
            s = self.cu_static[b]
            rows += list(range(s if mask == "beyond_alt" else s + r[0], s + r[0] + r[3]))
        self.cached = torch.tensor(rows, device="cuda", dtype=torch.long)
        self.ref_shape = (len(rows), heads, dim)
        self.scale = 1.0 / math.sqrt(dim)
        q, k, v, _ = self.static
        self.cache.build(0, q, k, v, torch.empty_like(q))

    def step_ref(self, ref):
        """Exact o and lse of the step, and the gradients' references."""
        q, k, v, do = self.live
        o, lse = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
        c0 = 0
        for b, r in enumerate(self.reqs):
            a = slice(self.cu_live[b], self.cu_live[b + 1])
            nc = r[3] + (r[0] if self.mask == "beyond_alt" else 0)
            c = slice(c0, c0 + nc)
            c0 += nc
            if a.stop == a.start:
                continue
            kc, vc = self.static[1][self.cached[c]], self.static[2][self.cached[c]]
            o[a], lse[a] = ref.group(q[a], do[a], [(k[a], v[a], ("dk", a, k.shape), ("dv", a, k.shape)),
                                                   (kc, vc, ("dk_ref", c, self.ref_shape), ("dv_ref", c, self.ref_shape))],
                                     self.scale, ("dq", a, q.shape))
        return o, lse

    def build_ref(self, ref):
        q, k, v, do = self.static
        o, lse = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
        for b, r in enumerate(self.reqs):
            s, m, e = self.cu_static[b], self.cu_static[b] + r[0], self.cu_static[b + 1]
            groups = [(slice(s, m), slice(s, m)), (slice(m, e), slice(s, e))] if self.mask == "beyond_alt" else [(slice(s, e),) * 2]
            for rows, keys in groups:
                if rows.stop > rows.start:
                    o[rows], lse[rows] = ref.group(q[rows], do[rows], [(k[keys], v[keys], ("dk", keys, k.shape), ("dv", keys, k.shape))],
                                                   self.scale, ("dq", rows, q.shape))
        return o, lse

    def step_backward(self, o, lse, ref_grads=True, into=None, accumulate=False):
        q, k, v, do = self.live
        g = {n: torch.full_like(q, float("nan")) for n in ("dq", "dk", "dv")}
        if into is None and ref_grads:
            into = [torch.full(self.ref_shape, float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        g.update(zip(("dk_ref", "dv_ref"), into if ref_grads else (None, None)))
        self.cache.step_backward(0, q, k, v, o, lse, do, **g, accumulate=accumulate)
        return g

    def build_backward(self, o, lse, dk_ref=None, dv_ref=None):
        q, k, v, do = self.static
        g = {n: torch.full_like(q, float("nan")) for n in ("dq", "dk", "dv")}
        self.cache.build_backward(0, q, k, v, o, lse, do, **g, dk_ref=dk_ref, dv_ref=dv_ref)
        return g


CASES = [
    (2, 64, [(3, 1, 1, 1)], "beyond"),  # one row of each kind
    (3, 128, [(0, 0, 1, 1)], "beyond"),
    (4, 64, [(32, 64, 256, 256)], "beyond"),
    (2, 128, [(13, 40, 217, 301), (0, 0, 130, 127), (7, 0, 0, 65), (5, 3, 254, 0)], "beyond"),  # no live rows; no references
    (2, 128, [(13, 40, 217, 301), (128, 1, 127, 129), (0, 5, 60, 257)], "beyond_alt"),
    (2, 64, [(77, 30, 153, 204), (13, 40, 77, 102), (64, 0, 1, 64)], "beyond_alt"),
    (3, 64, [(0, 64, 193, 385), (0, 0, 64, 1)], "isolated"),
    (1, 128, [(100, 100, 412, 1000)], "beyond"),
]


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"h{c[0]}d{c[1]}x{len(c[2])}{c[3]}")
def test_step_and_build_gradients(case, kernel):
    c = Case(*case, gain=2.0)
    rcb.set_kernel(kernel)
    ref = Ref()
    o, lse = c.step_ref(ref)
    got = c.step_backward(o.to(torch.bfloat16), lse.float())
    for n, t in got.items():
        ref.check(n, t)
    without = c.step_backward(o.to(torch.bfloat16), lse.float(), ref_grads=False)
    for n in ("dq", "dk", "dv"):
        assert torch.equal(got[n], without[n]), n
    ref = Ref()
    o, lse = c.build_ref(ref)
    o, lse = o.to(torch.bfloat16), lse.float()
    for n, t in c.build_backward(o, lse).items():
        ref.check(n, t)
    add = {n: torch.zeros_like(c.static[0]) for n in ("dk", "dv")}
    for n in add:
        add[n][c.cached] = got[n + "_ref"]
    for n, t in c.build_backward(o, lse, got["dk_ref"], got["dv_ref"]).items():
        ref.check(n, t, add.get(n))


def test_accumulated_reference_gradients():
    """Two steps that share a cache: the second call's sum is rounded once more."""
    c = Case(2, 128, [(8, 16, 200, 300)])
    ref = Ref()
    o, lse = c.step_ref(ref)
    first = c.step_backward(o.to(torch.bfloat16), lse.float())
    into = [first["dk_ref"].clone(), first["dv_ref"].clone()]
    c.step_backward(o.to(torch.bfloat16), lse.float(), into=into, accumulate=True)
    for n, t in zip(("dk_ref", "dv_ref"), into):
        ref.check(n, t, extra=first[n])


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dim", [64, 128])
def test_full_gradients_after_the_forward_call(dim, kernel):
    """o and lse as full_attention leaves them."""
    cu, H = [0, 1, 1, 258, 771], 2
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    q, k, v, do = (rnd(gen, cu[-1], H, dim) for _ in range(4))
    o, lse = torch.empty_like(q), torch.empty(cu[-1], H, device="cuda")
    rcb.full_attention(cu, q, k, v, o, lse)
    ref = Ref(forward=True)
    for a, b in zip(cu, cu[1:]):
        if b > a:
            r = slice(a, b)
            ref.group(q[r], do[r], [(k[r], v[r], ("dk", r, q.shape), ("dv", r, q.shape))], 1 / math.sqrt(dim), ("dq", r, q.shape))
    rcb.set_kernel(kernel)
    g = {n: torch.full_like(q, float("nan")) for n in ("dq", "dk", "dv")}
    rcb.full_attention_backward(cu, q, k, v, o, lse, do, **g)
    for n, t in g.items():
        ref.check(n, t)


def test_gradient_against_differences():
    """The sum of o . do along a direction of all inputs, differenced in 64 bits."""
    c = Case(2, 64, [(5, 7, 60, 90)], gain=1.5)
    ref = Ref()
    o, lse = c.step_ref(ref)
    got = c.step_backward(o.to(torch.bfloat16), lse.float())
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    q, k, v, do = (t.double() for t in c.live)
    kc, vc = (t[c.cached].double() for t in c.static[1:3])
    names = ("dq", "dk", "dv", "dk_ref", "dv_ref")
    x = [q, k, v, kc, vc]
    d = [torch.randn(t.shape, generator=gen, device="cuda", dtype=torch.float64) for t in x]

    def loss(h):
        q, k, v, kc, vc = (a + h * b for a, b in zip(x, d))
        keys, vals = torch.cat((k, kc)).transpose(0, 1), torch.cat((v, vc)).transpose(0, 1)
        p = torch.softmax(q.transpose(0, 1) @ keys.transpose(1, 2) * c.scale, -1)
        return ((p @ vals).transpose(0, 1) * do).sum()

    h = 1e-4
    slope = ((loss(h) - loss(-h)) / (2 * h)).item()
    along = sum((got[n].double() * t).sum() for n, t in zip(names, d)).item()
    bound = sum((ref.sums[n][1] * t.abs()).sum() for n, t in zip(names, d)).item()
    assert abs(along - slope) <= bound + 1e-5 * abs(slope)


def test_gradients_are_reproducible_and_alone_as_in_a_batch():
    reqs = [(13, 40, 217, 301), (64, 30, 512, 640), (0, 0, 130, 127)]
    c = Case(3, 128, reqs)
    o, lse = c.step_ref(Ref())
    o, lse = o.to(torch.bfloat16), lse.float()
    first, again = c.step_backward(o, lse), c.step_backward(o, lse)
    for n in first:
        assert torch.equal(first[n], again[n]), n
    one = Case(3, 128, reqs[1:2])
    live, cached = slice(c.cu_live[1], c.cu_live[2]), slice(301, 941)
    one.live = [t[live].contiguous() for t in c.live]
    st = slice(c.cu_static[1], c.cu_static[2])
    one.static = [t[st].contiguous() for t in c.static]
    one.cache.build(0, *one.static[:3], torch.empty_like(one.static[0]))
    alone = one.step_backward(o[live].contiguous(), lse[live].contiguous())
    for n, t in alone.items():
        assert torch.equal(t, first[n][cached if n.endswith("ref") else live]), n


def test_many_requests():
    """More requests than one launch's list holds (32)."""
    gen = torch.Generator().manual_seed(5)
    reqs = [tuple(int(x) for x in torch.randint(0, 40, (4,), generator=gen)) for _ in range(75)]
    c = Case(2, 64, reqs)
    ref = Ref()
    o, lse = c.step_ref(ref)
    for n, t in c.step_backward(o.to(torch.bfloat16), lse.float()).items():
        ref.check(n, t)


@pytest.mark.parametrize("kernel", KERNELS)
def test_no_live_rows_at_all(kernel):
    """Cached rows that no query sees: zeros, or what was there."""
    rcb.set_kernel(kernel)
    c = Case(2, 128, [(7, 0, 0, 300), (0, 0, 0, 1)])
    o, lse = torch.empty(0, 2, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 2, device="cuda")
    g = c.step_backward(o, lse)
    assert (g["dk_ref"] == 0).all() and (g["dv_ref"] == 0).all()
    held = [rnd(torch.Generator(device="cuda"), *c.ref_shape) for _ in range(2)]
    into = [t.clone() for t in held]
    c.step_backward(o, lse, into=into, accumulate=True)
    assert all(torch.equal(a, b) for a, b in zip(into, held))


def test_large_scores_and_zero_gradients():
    """Scores of hundreds (P is one-hot, its other weights underflow), and a do of zeros."""
    c = Case(2, 128, [(4, 8, 150, 200)], gain=40.0)
    o, lse = c.step_ref(Ref())
    got = c.step_backward(o.to(torch.bfloat16), lse.float())
    assert all(torch.isfinite(t).all() for t in got.values())
    c.live[3].zero_()
    assert all((t == 0).all() for t in c.step_backward(o.to(torch.bfloat16), lse.float()).values())


def test_other_stream_and_graph():
    c = Case(2, 128, [(16, 30, 300, 400)])
    o, lse = c.step_ref(Ref())
    o, lse = o.to(torch.bfloat16), lse.float()
    want = c.step_backward(o, lse)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    q, k, v, do = c.live
    g = {n: torch.zeros_like(t) for n, t in want.items()}
    torch.cuda.synchronize()
    c.cache.step_backward(0, q, k, v, o, lse, do, **g, stream=side)
    side.synchronize()
    for n in want:
        assert torch.equal(g[n], want[n]), n
    for t in g.values():
        t.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.step_backward(0, q, k, v, o, lse, do, **g)
    graph.replay()
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(g[n], want[n]), n


def test_refusals():
    c = Case(2, 128, [(4, 8, 20, 30)])
    o, lse = c.step_ref(Ref())
    o, lse = o.to(torch.bfloat16), lse.float()
    q, k, v, do = c.live
    out = [torch.empty_like(q) for _ in range(3)]
    ref = [torch.empty(c.ref_shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    with pytest.raises(ValueError, match="lse"):
        c.cache.step_backward(0, q, k, v, o, None, do, *out)
    with pytest.raises(ValueError, match="lse"):
        c.cache.step_backward(0, q, k, v, o, lse.double(), do, *out)
    with pytest.raises(ValueError, match="d_o"):
        c.cache.step_backward(0, q, k, v, o, lse, do.float(), *out)
    with pytest.raises(ValueError, match="dv_ref"):
        c.cache.step_backward(0, q, k, v, o, lse, do, *out, dk_ref=ref[0])
    with pytest.raises(rcb.RefCacheError, match="layer"):
        c.cache.step_backward(1, q, k, v, o, lse, do, *out)
    with pytest.raises(rcb.RefCacheError, match="scale"):
        c.cache.step_backward(0, q, k, v, o, lse, do, *out, scale=0.0)
    fresh = rcb.RefCache(c.seg)
    with pytest.raises(rcb.RefCacheError, match="built"):
        fresh.step_backward(0, q, k, v, o, lse, do, *out)
    e4m3 = rcb.RefCache(c.seg, cache_dtype="fp8")
    e4m3.build(0, *c.static[:3], torch.empty_like(c.static[0]))
    with pytest.raises(rcb.RefCacheError, match="bf16 cache"):
        e4m3.step_backward(0, q, k, v, o, lse, do, *out)


def test_workload_through_forward_and_backward():
    """The 512x512 two-reference edit at two heads' sample of its gradients."""
    w = workloads.EDIT_512_2REF
    r = w.requests[0]
    c = Case(2, w.head_dim, [(r.n_st, r.n_lt, r.n_x, r.n_r)])
    q, k, v, do = c.live
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    c.cache.step(0, q, k, v, o, lse)
    ref = Ref(forward=True)
    c.step_ref(ref)
    for n, t in c.step_backward(o, lse).items():
        ref.check(n, t)
