"""The linear layers of a block in 8 bits, and their inputs kept in 8 bits for the backward pass, as a user's program calls them.

The 8-bit form of a row is E4M3 codes and, for each 128 of its columns, a power of two as scale: the smallest with which
the largest magnitude stays within 448.  A weight's has one scale for each 128 x 128.

A case is one pass through one operator:

``rows``, ``weight``
    The 8-bit form of ``rows`` activations of ``k`` columns; of a weight [n, k], as it lies and transposed.
``linear``
    y = x w^T + bias from the 8-bit forms of x [rows, k] and w [n, k]; with ``transposed`` y = x w from x [rows, n].
``gelu_fwd``, ``gelu_bwd``
    The first linear layer of an MLP with the GELU behind it: its output and, as the checkpoint, its argument u, both in
    8 bits.  And the gradient: da = dy w2 from the second layer's weight w2 [k, n], du = da gelu'(u), in bf16 and in 8 bits.
``wgrad``
    The weight's gradient dy^T x from bf16 dy [rows, n] and the 8-bit x [rows, k], added to what earlier micro-batches
    gave, and the bias's.
"""
import math

import torch

own = False

BLOCK, LARGEST = 128, 448.0
TANH_A, TANH_B = math.sqrt(2.0 / math.pi), 0.044715

#: A drawn case's work stays below these (the largest listed cases do as much).
MOST_FLOPS, MOST_BYTES = 2.0e12, 4.0e8


def _case(name, op, rows, n, k, **more):
    c = {"op": op, "rows": rows, "n": n, "k": k, **more}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a toy model's live rows on their way into a projection
        _case("rows_tiny", "rows", 320, 0, 256),
        # the static rows of five 1024x1024 references, once a request and layer
        _case("rows_1024_5ref", "rows", 20608, 0, 4096),
        # an MLP's fp32 master weight behind the optimiser's step
        _case("weight_mlp", "weight", 0, 16384, 4096, dtype="fp32"),
        # shift, scale and gate of a block's two halves for the two branches of a guided step: one row each
        _case("linear_mod_cfg", "linear", 2, 24576, 4096, transposed=False, bias=True),
        # a toy model's fused projection
        _case("linear_tiny", "linear", 320, 768, 256, transposed=False, bias=False),
        # the fused projection of a 512x512 edit's live rows
        _case("linear_qkv_512", "linear", 1280, 12288, 4096, transposed=False, bias=True),
        # the input's gradient of that projection over the static rows of five 1024x1024 references
        _case("linear_dx_1024_5ref", "linear", 20608, 12288, 4096, transposed=True, bias=False),
        # the MLP of three requests of odd lengths, of a width that is no multiple of the blocks
        _case("gelu_fwd_odd", "gelu_fwd", 1777, 8240, 2064, form="erf", bias=True),
        # training on one 1024x1024 edit
        _case("gelu_bwd_1024", "gelu_bwd", 4608, 16384, 4096, form="tanh", bias=False),
        # a toy model's layer, odd sizes
        _case("wgrad_tiny_odd", "wgrad", 333, 272, 208, dtype="bf16", add=False, bias=False),
        # the fused projection of a 512x512 edit, adding to the micro-batches before
        _case("wgrad_qkv_512", "wgrad", 1280, 12288, 4096, dtype="fp32", add=True, bias=True),
        # the MLP of a 1024x1024 edit
        _case("wgrad_mlp_1024", "wgrad", 4608, 16384, 4096, dtype="fp32", add=False, bias=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rows", "weight", "linear", "linear", "linear", "gelu_fwd", "gelu_bwd", "wgrad", "wgrad"])
    while True:
        rows, n, k = _log_int(rng, 1, 20608), 16 * _log_int(rng, 8, 1024), 16 * _log_int(rng, 8, 1024)
        if op == "rows":
            c = _case("", op, rows, 0, k)
        elif op == "weight":
            c = _case("", op, 0, n, k, dtype=rng.choice(["fp32", "bf16"]))
        elif op == "linear":
            c = _case("", op, rows, n, k, transposed=rng.random() < 0.4, bias=rng.random() < 0.5)
        elif op == "wgrad":
            c = _case("", op, rows, n, k, dtype=rng.choice(["fp32", "fp32", "bf16"]), add=rng.random() < 0.5, bias=rng.random() < 0.3)
        else:
            c = _case("", op, rows, n, k, form=rng.choice(["tanh", "erf"]), bias=op == "gelu_fwd" and rng.random() < 0.5)
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return c


def work(case):
    r, n, k, op = case["rows"], case["n"], case["k"], case["op"]
    f8 = lambda rows, width: rows * (width + -(-width // BLOCK))  # noqa: E731
    if op == "rows":
        return {"bytes": 2 * r * k + f8(r, k), "flops": 3 * r * k}
    if op == "weight":
        return {"bytes": n * k * ((4 if case["dtype"] == "fp32" else 2) + 2), "flops": 3 * n * k}
    flops = 2 * r * n * k
    if op == "linear":
        i, o = (n, k) if case["transposed"] else (k, n)
        return {"bytes": f8(r, i) + n * k + 2 * r * o + (2 * o if case["bias"] else 0), "flops": flops}
    if op == "gelu_fwd":
        return {"bytes": f8(r, k) + n * k + 2 * f8(r, n) + (2 * n if case["bias"] else 0), "flops": flops}
    if op == "gelu_bwd":
        return {"bytes": f8(r, k) + n * k + 2 * f8(r, n) + 2 * r * n, "flops": flops}
    size = 4 if case["dtype"] == "fp32" else 2
    return {"bytes": 2 * r * n + f8(r, k) + n * k * size * (2 if case["add"] else 1), "flops": flops}


# ---------------------------------------------------------------- what a program holds before the call
def _inputs(case, seed):
    """The tensors in bf16 (a master weight: fp32) that the 8-bit forms are made of."""
    gen, r, n, k, op = torch.Generator(device="cuda"), case["rows"], case["n"], case["k"], case["op"]
    gen.manual_seed(int(seed))
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    # activations: channels of different size, a few of them large
    rows = lambda c, gain=1.0: (randn(r, c) * torch.exp(0.6 * randn(c)) * gain).to(torch.bfloat16)  # noqa: E731
    bias = lambda c: (0.1 * randn(c)).to(torch.bfloat16) if case["bias"] else None  # noqa: E731
    if op == "rows":
        return {"x": rows(k)}
    if op == "weight":
        return {"w": (randn(n, k) * k ** -0.5).to(torch.float32 if case["dtype"] == "fp32" else torch.bfloat16)}
    if op == "wgrad":
        x = {"dy": rows(n, 1e-3), "x": rows(k)}
        if case["add"]:
            x["add"] = (randn(n, k) * 1e-2).to(torch.float32 if case["dtype"] == "fp32" else torch.bfloat16)
        return x
    if op == "gelu_bwd":
        return {"x": rows(k, 1e-3), "w": (randn(k, n) * n ** -0.5).to(torch.bfloat16), "u": (1.5 * randn(r, n)).to(torch.bfloat16)}
    i, o = (n, k) if op == "linear" and case["transposed"] else (k, n)
    return {"x": rows(i), "w": (randn(n, k) * i ** -0.5).to(torch.bfloat16), "bias": bias(o)}


def _quantize(x, tall=1):
    """Codes [rows, width] and scales' exponents (uint8, biased by 127) [blocks of `tall` rows, blocks] of the 8-bit form."""
    r, c = x.shape
    rb, cb = -(-r // tall), -(-c // BLOCK)
    x = x.float()
    full = torch.nn.functional.pad(x, (0, cb * BLOCK - c, 0, rb * tall - r)).view(rb, tall, cb, BLOCK)
    m, e = torch.frexp(full.abs().amax((1, 3)))
    b = torch.where(m > 0, e + 118 + (m > LARGEST / 512).int(), 127).clamp(1, 254)
    codes = (full * torch.exp2(127.0 - b)[:, None, :, None]).view(rb * tall, cb * BLOCK)[:r, :c].to(torch.float8_e4m3fn)
    return codes, b.to(torch.uint8)


def _value(codes, b, tall=1):
    """The values that an 8-bit form stands for, in 32 bits."""
    r, c = codes.shape
    scale = torch.exp2(b.float() - 127.0).repeat_interleave(tall, 0)[:r].repeat_interleave(BLOCK, 1)[:, :c]
    return codes.float() * scale


def prepare(case, seed):
    x, op, r, n, k = _inputs(case, seed), case["op"], case["rows"], case["n"], case["k"]
    new = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    st = {"case": case, "in": x}
    if op == "linear":
        st["y"] = new(r, k if case["transposed"] else n)
    elif op == "gelu_bwd":
        st["du"] = new(r, n)
    elif op == "wgrad":
        st["dw"] = new(n, k, dtype=torch.float32 if case["dtype"] == "fp32" else torch.bfloat16)
        st["db"] = new(n, dtype=torch.float32) if case["bias"] else None
    if own:
        from paper_2608_21229_gb300 import refcache as rc

        st["rc"] = rc
        if op not in ("rows", "weight"):
            st["x8"] = rc.f8_quantize(x["x"])
            st["w8"] = rc.f8_quantize_weight(x["w"]) if "w" in x else None
            st["u8"] = rc.f8_quantize(x["u"]) if "u" in x else None
        st["out"] = rc.F8Weight(n, k) if op == "weight" else [rc.F8Rows(r, k if op == "rows" else n) for _ in range(2)]
    elif op not in ("rows", "weight"):
        st["x8"] = _quantize(x["x"])
        st["w8"] = _quantize(x["w"], BLOCK) if "w" in x else None
        st["u8"] = _quantize(x["u"]) if "u" in x else None
    return st


# ---------------------------------------------------------------- one pass
def _powers(b):
    return b.view(torch.float8_e8m0fnu)


def _form(codes, b):
    return {"codes": codes, "scales": _powers(b)}


def _gelu(u, form):
    """gelu(u) and its derivative."""
    if form == "erf":
        phi = 0.5 * (1.0 + torch.erf(u * math.sqrt(0.5)))
        return u * phi, phi + u * torch.exp(-0.5 * u * u) * math.sqrt(0.5 / math.pi)
    t = torch.tanh(TANH_A * (u + TANH_B * u * u * u))
    return 0.5 * u * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * u * (1.0 - t * t) * TANH_A * (1.0 + 3.0 * TANH_B * u * u)


def _run(st):
    case, x, op = st["case"], st["in"], st["case"]["op"]
    if op == "rows":
        return _form(*_quantize(x["x"]))
    if op == "weight":
        codes, b = _quantize(x["w"], BLOCK)
        return {**_form(codes, b), "codes_t": codes.t().contiguous(), "scales_t": _powers(b.t().contiguous())}
    x8 = _value(*st["x8"])
    if op == "wgrad":
        g = x["dy"].float().t() @ x8
        st["dw"].copy_(g + x["add"].float() if case["add"] else g)
        if case["bias"]:
            st["db"].copy_(x["dy"].float().sum(0))
        return {"dw": st["dw"], "db": st["db"]}
    w8 = _value(*st["w8"], BLOCK)
    if op == "gelu_bwd":
        du = (x8 @ w8) * _gelu(_value(*st["u8"]), case["form"])[1]
        st["du"].copy_(du)
        return {"du": st["du"], "du8": _form(*_quantize(du))}
    u = x8 @ (w8 if op == "linear" and case["transposed"] else w8.t())
    if case["bias"]:
        u = u + x["bias"].float()
    if op == "linear":
        st["y"].copy_(u)
        return st["y"]
    return {"a8": _form(*_quantize(_gelu(u, case["form"])[0])), "u8": _form(*_quantize(u))}


def _parts(x8):
    return {"codes": x8.codes, "scales": x8.scales}


def _run_own(st):
    rc, case, x, op = st["rc"], st["case"], st["in"], st["case"]["op"]
    if op == "rows":
        return _parts(rc.f8_quantize(x["x"], st["out"][0]))
    if op == "weight":
        w = rc.f8_quantize_weight(x["w"], st["out"])
        return {**_parts(w), "codes_t": w.codes_t, "scales_t": w.scales_t}
    if op == "wgrad":
        rc.f8_weight_grad(x["dy"], st["x8"], st["dw"], add=x.get("add"), d_bias=st["db"])
        return {"dw": st["dw"], "db": st["db"]}
    if op == "linear":
        rc.f8_linear(st["x8"], st["w8"], st["y"], bias=x["bias"], transposed=case["transposed"])
        return st["y"]
    if op == "gelu_fwd":
        a8, u8 = st["out"]
        rc.f8_linear_gelu(st["x8"], st["w8"], a8, u8, bias=x["bias"], form=case["form"])
        return {"a8": _parts(a8), "u8": _parts(u8)}
    rc.f8_linear_gelu_backward(st["x8"], st["w8"], st["u8"], st["du"], st["out"][0], form=case["form"])
    return {"du": st["du"], "du8": _parts(st["out"][0])}


def run(st):
    return _run_own(st) if own else _run(st)


# ---------------------------------------------------------------- the same in 64 bits
def _grid(x, tall=1):
    """The 8-bit form by the formats' definitions: (codes' values, scales) in 64 bits, the scales [blocks, blocks]."""
    r, c = x.shape
    x = x.double()
    rb, cb = -(-r // tall), -(-c // BLOCK)
    amax = torch.zeros(rb, c, dtype=torch.float64, device="cuda").index_reduce_(0, torch.arange(r, device="cuda") // tall, x.abs(), "amax")
    amax = torch.zeros(rb, cb, dtype=torch.float64, device="cuda").index_reduce_(1, torch.arange(c, device="cuda") // BLOCK, amax, "amax")
    scale = torch.exp2(torch.ceil(torch.log2(amax / LARGEST)))
    scale = torch.where(scale * LARGEST < amax, 2 * scale, torch.where(scale * (LARGEST / 2) >= amax, scale / 2, scale))
    scale = torch.where(amax > 0, scale, 1.0).clamp(2.0 ** -126, 2.0 ** 127)
    y = x / _spread(scale, r, c, tall)
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(y / unit) * unit, scale


def _spread(scale, r, c, tall):
    return scale.repeat_interleave(tall, 0)[:r].repeat_interleave(BLOCK, 1)[:, :c]


def _meant(x, tall=1):
    codes, scale = _grid(x, tall)
    return codes * _spread(scale, *x.shape, tall)


def _pair(x):
    codes, scale = _grid(x)
    return {"codes": codes, "scales": scale}


def exact(case, seed):
    x, op = _inputs(case, seed), case["op"]
    if op == "rows":
        return _pair(x["x"])
    if op == "weight":
        codes, scale = _grid(x["w"], BLOCK)
        return {"codes": codes, "scales": scale, "codes_t": codes.t(), "scales_t": scale.t()}
    a = _meant(x["x"])
    if op == "wgrad":
        g, dy = 0.0, x["dy"].double()
        for at in range(0, case["rows"], 8192):
            g = g + torch.einsum("rn,rk->nk", dy[at:at + 8192], a[at:at + 8192])
        return {"dw": g + x["add"].double() if case["add"] else g, "db": torch.einsum("rn->n", dy) if case["bias"] else None}
    w = _meant(x["w"], BLOCK)
    if op == "gelu_bwd":
        u = _meant(x["u"]).requires_grad_()
        g = torch.nn.functional.gelu(u, approximate="tanh" if case["form"] == "tanh" else "none")
        du = torch.autograd.grad(g, u, torch.einsum("rk,kn->rn", a, w))[0]
        return {"du": du, "du8": _pair(du)}
    y = torch.einsum("rn,nk->rk" if op == "linear" and case["transposed"] else "rk,nk->rn", a, w)
    if case["bias"]:
        y = y + x["bias"].double()
    if op == "linear":
        return y
    return {"a8": _pair(torch.nn.functional.gelu(y, approximate="tanh" if case["form"] == "tanh" else "none")), "u8": _pair(y)}
