"""The parameters' gradients of gated_norm against sums in 64 bits, each column within a bound of its own terms, so
that a block's sum that is lost or taken twice is seen: one row less would be.

Bounds, in units of E = 2^-24 of fp32's roundings.  A sum of n terms in fp32 is off by at most its depth times E of the sum
of their sizes: a block's rows (at most 16 here), its slots one after the other or in groups with 16 warps (at most 64), the
requests (at most 64 a launch): SUM = 160.  A row's mean and deviation come from sums of at most 16 columns a thread and 10
exchanges: 26 E of the mean size each, so xhat = (x - mean) / deviation is off by at most 64 E (|xhat| + 1), with its own
roundings (the mean is below a deviation here).  The gradient of the stream, d = dx_out + (u - mean(u) - xhat mean(u xhat)) /
deviation, has terms of sizes that add up to D below, each off by at most 128 E of itself."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

import test_gpu_block_ops as block
from test_gpu_block_ops import BF16, IDS, NormCase

pytestmark = pytest.mark.gpu

E, SUM, STAT, GRAD = 2.0 ** -24, 160, 64, 128


def normalised(t, kind):
    """The normalised rows, and the factor that takes a row's distances to them."""
    if kind is None:
        return t, torch.ones_like(t[:, :1])
    c = t - t.mean(-1, keepdim=True) if kind == "layer" else t
    r = (c.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
    return c * r, r


def gradients(c, **got):
    f32 = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    got = {"d_gate": f32(c.B, c.width), "d_scale": f32(c.B, c.width), "d_shift": f32(c.B, c.width)}
    got.update({"d_" + n: f32(c.width) for n, t in c.w.items() if t is not None})
    mods = {n: c.mods[n] for n in ("gate", "scale")}
    rcb.gated_norm_backward(c.cu, c.x, c.dy, torch.empty_like(c.x), branch=c.branch, dx_out=c.dx_out, **mods, **c.w, **c.kw, **got)
    return got


def by_request(c, rows):
    out = torch.zeros(c.B, c.width, dtype=torch.float64, device="cuda")
    return out.index_add_(0, c.req, rows)


@pytest.mark.parametrize("case", [
    ([1], 8, "layer", None, BF16, False),
    ([3, 0, 2], 64, "rms", "rms", torch.float32, True),
    ([5, 130, 1], 1000, "layer", "layer", BF16, True),
    ([40, 0, 7], 24 * 128, "layer", "rms", torch.float32, True),
    ([900], 256, None, "rms", BF16, False),
    ([17, 5], 8192, "layer", "rms", BF16, True),
    ([2] * 70 + [0, 9], 512, "rms", None, BF16, True),  # more requests than one launch takes
    ([70, 0, 95], 200, "rms", None, BF16, False),  # many slots a request, each request by itself
    ([3] * 40, 136, "layer", "rms", torch.float32, False),  # few
    ([9] * 40, 136, "layer", None, torch.float32, True),  # few, added up over the requests
    ([1500, 1, 900], 2056, "rms", "rms", BF16, True),  # blocks that take several rows and go on to the next request
    ([1100, 1300], 1032, "layer", "layer", BF16, False),
    ([333, 500, 1, 0, 777] * 3, 2048, "layer", "rms", BF16, True),  # the same with few slots a request
], **IDS)
def test_sums_within_their_terms(case):
    c = NormCase(*case)
    got = gradients(c)
    x, f, dy, dxo = (t.double() for t in (c.x, c.branch, c.dy, c.dx_out))
    one = torch.ones(c.width, dtype=torch.float64, device="cuda")
    w, pw = (one if t is None else t.double() for t in c.w.values())
    gate, scale = (c.mods[n].double() for n in ("gate", "scale"))
    xhat, r = normalised(x, c.kw["norm"])
    fhat, _ = normalised(f, c.kw["post_norm"])
    u = dy * (1 + scale[c.req]) * w
    m1 = u.mean(-1, keepdim=True) if c.kw["norm"] == "layer" else torch.zeros_like(r)
    m2 = (u * xhat).mean(-1, keepdim=True) if c.kw["norm"] else torch.zeros_like(r)
    d = dxo + r * (u - m1 - xhat * m2)
    sizes = u.abs()
    if c.kw["norm"]:
        sizes = sizes + u.abs().mean(-1, keepdim=True) + (1 + xhat.abs()) * (u.abs() * (1 + xhat.abs())).mean(-1, keepdim=True)
    D = dxo.abs() + r * sizes
    # each row's term, and what it may be off by without the sum
    terms = {"A": (dy, 0 * dy, dy.abs()), "B": (dy * xhat, STAT * dy.abs() * (xhat.abs() + 1), (dy * xhat).abs()),
             "G": (d * fhat, (GRAD + STAT) * D * (fhat.abs() + 1), (d * fhat).abs())}
    for name, kind, per, over in (("d_shift", "A", one, None), ("d_scale", "B", w, "d_weight"), ("d_gate", "G", pw, "d_post_weight")):
        val, off, size = terms[kind]
        bound = E * (by_request(c, off) + SUM * by_request(c, size) + 4 * by_request(c, val).abs())
        factor = {"d_weight": 1 + scale, "d_post_weight": gate}.get(over)
        results = [(name, by_request(c, val) * per, bound * per.abs(), val * per)]
        if over in got:
            results.append((over, (by_request(c, val) * factor).sum(0), (bound * factor.abs()).sum(0) * (1 + SUM * E) +
                            SUM * E * (by_request(c, size) * factor.abs()).sum(0), val * factor[c.req]))
        for n, ref, b, rows in results:
            err = (got[n].double() - ref).abs()
            assert torch.isfinite(got[n]).all() and (err <= 1.01 * b + 1e-37).all(), f"{n}: {(err / b.clamp_min(1e-37)).max().item():.3g} of its bound"
            # a row that is missing, or there twice, would be seen
            room = b[c.req] if b.dim() == 2 else b
            seen = (rows.abs() > 2.1 * room).any(-1)
            assert seen.all(), f"{n}: {(~seen).sum().item()} of {c.n} rows could be lost unseen"


@pytest.mark.parametrize("lens,width", [
    ([4000], 136),  # many slots, blocks of four rows
    ([1500, 1, 0, 900], 2056),  # blocks of eight, which go on to the next request
    ([2] * 70 + [0, 90], 512),  # few slots, two launches
    ([333, 500, 1, 0, 777] * 3, 2048),
    ([40, 0, 7], 24 * 128),
], ids=lambda x: f"{len(x)}" if isinstance(x, list) else str(x))
def test_small_integers_are_summed_exactly(lens, width):
    """Without norms and with small integers every product and sum is a whole number below 2^24."""
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    ints = lambda lo, hi, *s: torch.randint(lo, hi + 1, s, generator=g, device="cuda").to(BF16)  # noqa: E731
    n, B = sum(lens), len(lens)
    cu = [sum(lens[:i]) for i in range(B + 1)]
    req = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(lens, device="cuda"))
    x, branch, dy, dxo = (ints(-4, 4, n, width) for _ in range(4))
    gate, scale, w = ints(-2, 2, B, width), ints(-2, 2, B, width), ints(-3, 3, width)
    f32 = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    got = {"d_gate": f32(B, width), "d_scale": f32(B, width), "d_shift": f32(B, width), "d_weight": f32(width)}
    rcb.gated_norm_backward(cu, x, dy, torch.empty_like(x), branch=branch, dx_out=dxo, gate=gate, scale=scale, weight=w, norm=None, **got)
    x, branch, dy, dxo, gate, scale, w = (t.double() for t in (x, branch, dy, dxo, gate, scale, w))
    add = lambda t: torch.zeros(B, width, dtype=torch.float64, device="cuda").index_add_(0, req, t)  # noqa: E731
    d = dxo + dy * (1 + scale[req]) * w
    want = {"d_gate": add(d * branch), "d_scale": add(dy * x) * w, "d_shift": add(dy), "d_weight": (add(dy * x) * (1 + scale)).sum(0)}
    for name, ref in want.items():
        assert torch.equal(got[name].double(), ref), name


@pytest.mark.parametrize("norm,post", [("layer", None), ("rms", "rms"), ("layer", "layer")])
def test_rows_of_24_heads_of_128(norm, post):
    """The width of the edit workloads' model, which leaves a quarter of a block's vectors empty."""
    block.test_gated_norm(([13, 0, 60], 24 * 128, norm, post, BF16, True))
    block.test_gated_norm_backward(([13, 0, 60], 24 * 128, norm, post, BF16, True))
