"""Guard bytes around every buffer that the gradients and the block operators write, their workspaces among them, as
test_gpu_canary.py has them around the forward calls': nothing is written beside an output, no element of one is left
out, and no input changes.  Requests end inside tiles, and some are empty."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

from test_gpu_backward import Case, Ref
from test_gpu_block_ops import NormCase, RopeCase
from test_gpu_canary import PATTERN, Guarded

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def works(monkeypatch):
    """Workspaces between guards, which are checked at the end of the test."""
    made = []

    def work(nbytes, like, stream):
        made.append(Guarded((max(16, nbytes),), torch.uint8))
        return made[-1].t

    monkeypatch.setattr(rcb, "_work", work)
    old = rcb.set_kernel("tcgen05")
    yield made
    rcb.set_kernel(old)
    torch.cuda.synchronize()
    assert rcb.status() == rcb.OK, rcb.last_error()
    for i, g in enumerate(made):
        g.check(f"workspace {i}", written=False)


class Inputs:
    def __init__(self, *tensors):
        self.pairs = [(t, t.clone()) for t in tensors if t is not None]

    def check(self):
        for t, before in self.pairs:
            assert torch.equal(t.view(torch.uint8) if t.is_contiguous() else t, before.view(torch.uint8) if t.is_contiguous() else before)


def guarded(**shapes):
    return {n: Guarded(s, dt) for n, (s, dt) in shapes.items()}


def check(outs):
    for n, g in outs.items():
        g.check(n)


ATTN = [
    (3, 128, [(13, 40, 217, 301), (0, 0, 130, 127), (7, 0, 0, 65), (5, 3, 254, 0), (3, 1, 0, 5)], "beyond"),
    (3, 128, [(13, 40, 217, 301), (128, 1, 127, 129), (0, 5, 60, 257)], "beyond_alt"),
    (3, 64, [(77, 30, 153, 204), (13, 40, 77, 102), (64, 0, 1, 64), (0, 0, 0, 0)], "beyond"),
    (3, 64, [(77, 30, 153, 204), (1, 0, 515, 64)], "beyond_alt"),
]


@pytest.mark.parametrize("kernel", ["tcgen05", "mma_sync"])
@pytest.mark.parametrize("case", ATTN, ids=lambda c: f"d{c[1]}{c[3]}")
def test_attention_gradients_write_their_outputs_only(case, kernel, works):
    c = Case(*case)
    rcb.set_kernel(kernel)
    o, lse = c.step_ref(Ref())
    o, lse = o.to(BF16), lse.float()
    slots = list(c.cache.kv(0))
    thd = lambda n: ((n, c.H, c.D), BF16)  # noqa: E731
    n = c.cu_live[-1]
    kept = Inputs(*c.live, o, lse, *slots)
    for accumulate in (False, True):
        g = guarded(dq=thd(n), dk=thd(n), dv=thd(n), dk_ref=(c.ref_shape, BF16), dv_ref=(c.ref_shape, BF16))
        if accumulate:
            for m in ("dk_ref", "dv_ref"):
                g[m].t.normal_()
        q, k, v, do = c.live
        c.cache.step_backward(0, q, k, v, o, lse, do, **{m: x.t for m, x in g.items()}, accumulate=accumulate)
        check(g)
    added = [g[m].t.clone() for m in ("dk_ref", "dv_ref")]
    kept.check()
    o, lse = c.build_ref(Ref())
    o, lse, n = o.to(BF16), lse.float(), c.cu_static[-1]
    kept = Inputs(*c.static, o, lse, *added, *slots)
    q, k, v, do = c.static
    for ref in ({}, dict(dk_ref=added[0], dv_ref=added[1])):
        g = guarded(dq=thd(n), dk=thd(n), dv=thd(n))
        c.cache.build_backward(0, q, k, v, o, lse, do, **{m: x.t for m, x in g.items()}, **ref)
        check(g)
    kept.check()
    # the static rows as packed sequences of their own
    g = guarded(dq=thd(n), dk=thd(n), dv=thd(n))
    rcb.full_attention(c.cu_static, q, k, v, o, lse)
    kept = Inputs(*c.static, o, lse)
    rcb.full_attention_backward(c.cu_static, q, k, v, o, lse, do, **{m: x.t for m, x in g.items()})
    check(g)
    kept.check()
    assert len(works) == 5


ROPE = [(37, 3, 128, (16, 56, 56), "interleaved", F32, 53), (301, 5, 64, (8, 28, 28), "halves", BF16, 200), (5003, 2, 64, (64,), "halves", None, None),
        (1, 24, 128, (16, 56, 56), "halves", BF16, None)]


def apart(rows, H, D, pad):
    """[rows, H, D] whose rows lie `pad` elements apart, inside guards."""
    g = Guarded((rows, H * D + pad), BF16)
    return g, g.t[:, :H * D].view(rows, H, D) if pad == 0 else g.t.as_strided((rows, H, D), (H * D + pad, D, 1))


@pytest.mark.parametrize("case", ROPE, ids=lambda c: "-".join(str(x) for x in c[:3]))
def test_qkv_rope_writes_its_outputs_only(case):
    c = RopeCase(*case)
    q, k, v = c.qkv.unbind(1)
    kept = Inputs(c.qkv, c.pos, c.rows, *c.w, *c.grads)
    n = len(c.qkv)
    outs = [Guarded((c.out_rows, c.H, c.D), BF16) for _ in range(3)]
    rcb.qkv_rope(c.rope, c.pos, q, k, v, *(g.t for g in outs), *c.w, rows=c.rows)
    hit = torch.zeros(c.out_rows, dtype=torch.bool, device="cuda")
    hit[c.to[c.kept]] = True
    bits = PATTERN * 0x101 - 0x10000
    for i, g in enumerate(outs):
        g.check(f"output {i}", written=False)
        rows = g.t.view(torch.int16).flatten(1)
        assert (rows[~hit] == bits).all() and (rows[hit] != bits).all()
    pad = 24
    grads = [apart(n, c.H, c.D, pad) for _ in range(3)]
    dw = [None if w is None else Guarded((c.D,), F32) for w in c.w]
    rcb.qkv_rope_backward(c.rope, c.pos, q, k, *c.grads, *(t for _, t in grads), *c.w, *(None if g is None else g.t for g in dw), rows=c.rows)
    for i, (g, t) in enumerate(grads):
        g.check(f"gradient {i}", written=False)
        assert (g.t[:, c.H * c.D:].view(torch.int16) == bits).all()  # between the rows
        assert (t.contiguous().view(torch.int16) != bits).all()
    for i, g in enumerate(dw):
        if g is not None:
            g.check(f"weight gradient {i}")
    kept.check()


NORM = [([1], 8, "layer", None, BF16, False), ([5, 130, 1], 1000, "layer", "layer", BF16, True), ([40, 0, 7], 4104, "layer", "rms", F32, True),
        ([2] * 70 + [0, 9], 512, "rms", None, BF16, True), ([1500, 1, 900], 2056, "rms", "rms", BF16, True), ([17, 5], 8192, "layer", "rms", BF16, True)]


@pytest.mark.parametrize("case", NORM, ids=lambda c: f"{len(c[0])}x{c[1]}")
def test_gated_norm_writes_its_outputs_only(case):
    c = NormCase(*case)
    kept = Inputs(c.x, c.branch, c.dy, c.dx_out, *c.mods.values(), *c.w.values())
    rows, per, vec = ((c.n, c.width), BF16), ((c.B, c.width), F32), ((c.width,), F32)
    g = guarded(x_out=rows, y=rows)
    rcb.gated_norm(c.cu, c.x, branch=c.branch, **{n: x.t for n, x in g.items()}, **c.mods, **c.w, **c.kw)
    check(g)
    g = guarded(dx=rows, d_branch=rows, d_gate=per, d_scale=per, d_shift=per)
    g.update(guarded(**{"d_" + n: vec for n, t in c.w.items() if t is not None}))
    rcb.gated_norm_backward(c.cu, c.x, c.dy, branch=c.branch, dx_out=c.dx_out, gate=c.mods["gate"], scale=c.mods["scale"], **c.w, **c.kw,
                            **{n: x.t for n, x in g.items()})
    check(g)
    kept.check()


@pytest.mark.parametrize("out32", [False, True])
def test_clip_gradients_writes_its_outputs_only(out32):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    sizes = [(1, BF16), (16385, F32), (70_003, BF16), (33, F32)] * 150  # more than one launch takes
    grads = [torch.randn(n, generator=gen, device="cuda").to(dt) for n, dt in sizes]
    kept = Inputs(*grads[:8])
    outs = [Guarded((n,), F32 if out32 else dt) for n, dt in sizes[:8]]
    rest = [torch.empty(n, dtype=dt, device="cuda") for n, dt in sizes[8:]]
    norm = Guarded((1,), F32)
    rcb.clip_gradients(grads, 0.05, out=[g.t for g in outs] + rest, norm=norm.t)
    for i, g in enumerate(outs + [norm]):
        g.check(f"output {i}")
    kept.check()
