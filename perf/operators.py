"""The operators of a training or serving block around the joint attention, as a user's program calls them.

A case is one pass through one operator:

``step_bwd``, ``build_bwd``, ``full_bwd``
    The gradients of one layer's attention call: a denoising step over the reference cache, the static prefill, and the
    full recompute of a teacher.  ``reqs`` lists the batch's requests as ``n_st,n_lt,n_x,n_r`` (anchor, instruction,
    target and reference tokens), ``;`` between requests; tensors are packed ``[tokens, heads, dim]`` bf16.
``rope_fwd``, ``rope_bwd``
    From the fused projection ``[tokens, 3, heads, dim]`` to the attention's q, k and v: RMS norm of each head's query
    and key, rotary positions on three axes (frame, y, x), rows moved from the streams' order (all text rows, then all
    image rows) to the packed requests'.  ``reqs`` is ``n_text,h,w,frames`` per request.
``norm_fwd``, ``norm_bwd``
    The end of one block's half and the start of the next: the residual stream plus the gated (and, with ``post``,
    normalised) branch, then the norm with the next half's scale and shift.  ``reqs`` lists the requests' rows.
``clip``
    The global norm of a model's gradients and the clipped gradients.
"""
import math

import torch

own = False

#: A drawn case's work stays below these (the largest listed cases of the kind do more).
MOST_FLOPS, MOST_PAIRS, MOST_BYTES = 2.4e12, 2.2e9, 1.2e9

AXES = {128: (16, 56, 56), 64: (8, 28, 28)}
THETA = 10000.0
EPS = 1e-6
MAX_NORM = 0.05


def _attn(name, kind, heads, dim, reqs, mask="beyond", gain=1.0, ref_grad=True):
    c = {"op": "attn", "kind": kind, "heads": heads, "dim": dim, "reqs": reqs, "mask": mask, "gain": gain, "ref_grad": ref_grad}
    return dict(c, name=name) if name else c


def _rope(name, kind, heads, dim, reqs, pairs="interleaved", norm=True, wdtype="bf16"):
    c = {"op": "rope", "kind": kind, "heads": heads, "dim": dim, "reqs": reqs, "pairs": pairs, "norm": norm, "wdtype": wdtype}
    return dict(c, name=name) if name else c


def _norm(name, kind, width, reqs, norm="layer", post="none", mods="bf16", weight=False):
    c = {"op": "norm", "kind": kind, "width": width, "reqs": reqs, "norm": norm, "post": post, "mods": mods, "weight": weight}
    return dict(c, name=name) if name else c


def _clip(name, width, layers, dtype="bf16", out="same", odd=False, gain=1e-3):
    c = {"op": "clip", "kind": "clip", "width": width, "layers": layers, "dtype": dtype, "out": out, "odd": odd, "gain": gain}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a toy model's training step: all launch and latency
        _attn("step_bwd_tiny_d64", "step_bwd", 4, 64, "32,64,256,256"),
        # distilling on 512x512 edits with two references: an ordinary step of one sample
        _attn("step_bwd_512_2ref", "step_bwd", 24, 128, "64,256,1024,2048", gain=2.5),
        # 1024x1024 with five references, the longest training sample
        _attn("step_bwd_1024_5ref", "step_bwd", 24, 128, "128,512,4096,20480"),
        # the static block of three requests of odd lengths at head dim 64, anchors that see anchors only, and the
        # gradients that the step gave to the cached rows
        _attn("build_bwd_odd_d64", "build_bwd", 16, 64, "77,301,1537,2049;13,40,777,1021;128,511,4095,6143", mask="beyond_alt"),
        # a toy model's projections
        _rope("rope_fwd_tiny", "rope_fwd", 4, 64, "64,16,16,1", wdtype="fp32"),
        # the static rows of five 1024x1024 references, once a request
        _rope("rope_fwd_1024_5ref", "rope_fwd", 24, 128, "128,64,64,5"),
        # the live rows of a 1024x1024 edit in training, pairs in halves
        _rope("rope_bwd_1024", "rope_bwd", 24, 128, "512,64,64,1", pairs="halves"),
        # a toy model's block
        _norm("norm_fwd_tiny", "norm_fwd", 256, "320"),
        # guided sampling at 1024x1024: the rows of both branches, each with its own modulation
        _norm("norm_fwd_1024_cfg", "norm_fwd", 4096, "4608;4096"),
        # training on two samples of different size, branch normalised before its gate
        _norm("norm_bwd_2req_post", "norm_bwd", 4096, "4608;1280", norm="rms", post="rms", mods="fp32", weight=True),
        # the gradients of one block of a toy model, odd sizes and offsets among them
        _clip("clip_tiny_odd", 256, 1, odd=True),
        # the gradients of a model of 0.9 billion parameters
        _clip("clip_model", 2048, 12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "rope", "rope", "norm", "norm", "clip"])
    while True:
        if op == "attn":
            kind = rng.choice(["step_bwd", "step_bwd", "build_bwd", "full_bwd"])
            mask = rng.choice(["beyond", "beyond", "beyond_alt", "isolated"]) if kind != "full_bwd" else "beyond"
            reqs = [(0 if mask == "isolated" else rng.randint(0, 128), rng.randint(0, 512), _log_int(rng, 100, 4608),
                     _log_int(rng, 100, 20480)) for _ in range(rng.choice([1, 1, 2, 3]))]
            c = _attn("", kind, _log_int(rng, 2, 32), rng.choice([128, 128, 64]), ";".join(",".join(map(str, r)) for r in reqs),
                      mask, rng.choice([1.0, 2.5]), rng.random() < 0.7)
        elif op == "rope":
            reqs = [(rng.randint(0, 512), _log_int(rng, 4, 64), _log_int(rng, 4, 64), rng.choice([1, 1, 2, 5]))
                    for _ in range(rng.choice([1, 1, 2, 3]))]
            c = _rope("", rng.choice(["rope_fwd", "rope_bwd"]), _log_int(rng, 2, 32), rng.choice([128, 128, 64]),
                      ";".join(",".join(map(str, r)) for r in reqs), rng.choice(["interleaved", "halves"]), rng.random() < 0.8,
                      rng.choice(["bf16", "fp32"]))
        elif op == "norm":
            c = _norm("", rng.choice(["norm_fwd", "norm_bwd"]), 8 * _log_int(rng, 8, 768),
                      ";".join(str(_log_int(rng, 1, 8192)) for _ in range(rng.choice([1, 2, 4]))), rng.choice(["layer", "rms"]),
                      rng.choice(["none", "rms", "layer"]), rng.choice(["bf16", "fp32"]), rng.random() < 0.5)
        else:
            c = _clip("", 8 * _log_int(rng, 16, 256), rng.randint(1, 8), rng.choice(["bf16", "bf16", "fp32"]),
                      rng.choice(["same", "fp32"]), rng.random() < 0.5, rng.choice([1e-3, 1e-7]))
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and (c["op"] != "attn" or _pairs(c) * c["heads"] <= MOST_PAIRS):
            return c


# ---------------------------------------------------------------- sizes
def _ints(case):
    return [tuple(int(n) for n in r.split(",")) for r in case["reqs"].split(";")]


def _cu(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _kept(case, r):
    return r[0] + r[3] if case["mask"] == "beyond_alt" else r[3]


def _groups(case):
    """The attention as groups of rows that see the same keys: (query rows, key rows of the call, rows of the cache)."""
    out, l0, s0, c0 = [], 0, 0, 0
    for r in _ints(case):
        live, static, kept = r[1] + r[2] + (r[3] if case["kind"] == "full_bwd" else 0), r[0] + r[3], _kept(case, r)
        if case["kind"] != "build_bwd":
            out.append((slice(l0, l0 + live), slice(l0, l0 + live), slice(c0, c0 + (kept if case["kind"] == "step_bwd" else 0))))
        elif case["mask"] == "beyond_alt":
            out.append((slice(s0, s0 + r[0]), slice(s0, s0 + r[0]), slice(0, 0)))
            out.append((slice(s0 + r[0], s0 + static), slice(s0, s0 + static), slice(0, 0)))
        else:
            out.append((slice(s0, s0 + static), slice(s0, s0 + static), slice(0, 0)))
        l0, s0, c0 = l0 + live, s0 + static, c0 + kept
    return [g for g in out if g[0].stop > g[0].start]


def _len(s):
    return s.stop - s.start


def _pairs(case):
    return sum(_len(q) * (_len(a) + _len(b)) for q, a, b in _groups(case))


def _rows(case):
    """Rows of the call's tensors, and of the cache."""
    reqs = _ints(case)
    if case["kind"] == "build_bwd":
        rows = sum(r[0] + r[3] for r in reqs)
    else:
        rows = sum(r[1] + r[2] + (r[3] if case["kind"] == "full_bwd" else 0) for r in reqs)
    return rows, sum(_kept(case, r) for r in reqs)


def _clip_shapes(case):
    """The parameters of ``layers`` blocks: projections, a two-matrix MLP, modulation, their biases and head norms."""
    c = case["width"]
    block = [(3 * c, c), (3 * c,), (c, c), (c,), (4 * c, c), (4 * c,), (c, 4 * c), (c,), (6 * c, c), (6 * c,)]
    if case["odd"]:
        block += [(c // 2 + 1,), (7, c + 3), (1,)]
    return block * case["layers"]


def work(case):
    if case["op"] == "attn":
        h, d = case["heads"], case["dim"]
        rows, cached = _rows(case)
        b = h * d * 2 * 8 * rows + 4 * h * rows  # q, k, v, o and the output's gradient read, dq, dk and dv written; log-sum-exp
        if case["kind"] == "step_bwd":
            b += h * d * 2 * (4 if case["ref_grad"] else 2) * cached
        elif case["kind"] == "build_bwd" and case["ref_grad"]:
            b += h * d * 2 * 2 * cached
        return {"bytes": b, "flops": 10 * d * h * _pairs(case)}
    if case["op"] == "rope":
        h, d, n = case["heads"], case["dim"], sum(r[0] + r[1] * r[2] * r[3] for r in _ints(case))
        moved = 6 if case["kind"] == "rope_fwd" else 8 if case["norm"] else 6
        return {"bytes": n * (moved * h * d * 2 + 16), "flops": n * h * d * (12 if case["kind"] == "rope_fwd" else 30)}
    if case["op"] == "norm":
        c, n, batch = case["width"], sum(int(r) for r in case["reqs"].split(";")), len(case["reqs"].split(";"))
        m = 2 if case["mods"] == "bf16" else 4
        fwd = case["kind"] == "norm_fwd"
        # forward: stream, branch read, stream and normed row written; backward: stream, branch, two gradients read, two written
        return {"bytes": n * c * 2 * (4 if fwd else 6) + batch * c * (3 * m if fwd else 2 * m + 12), "flops": n * c * (12 if fwd else 30)}
    n = sum(math.prod(s) for s in _clip_shapes(case))
    size = 2 if case["dtype"] == "bf16" else 4
    return {"bytes": n * (size + (size if case["out"] == "same" else 4)), "flops": 3 * n}


# ---------------------------------------------------------------- what a program holds before the call
def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _randn(gen, shape, gain=1.0, mean=0.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * gain + mean).to(dtype)


def _heads_first(x):
    return x.transpose(0, 1).float()


def _attn_inputs(case, seed):
    gen, h, d = _gen(seed), case["heads"], case["dim"]
    rows, cached = _rows(case)
    x = {"q": _randn(gen, (rows, h, d), case["gain"])}
    for n in ("k", "v", "do"):
        x[n] = _randn(gen, (rows, h, d))
    if case["kind"] == "step_bwd":
        x["kc"], x["vc"] = _randn(gen, (cached, h, d)), _randn(gen, (cached, h, d))
    elif case["kind"] == "build_bwd" and case["ref_grad"]:
        x["dk_ref"], x["dv_ref"] = _randn(gen, (cached, h, d), 0.1), _randn(gen, (cached, h, d), 0.1)
    return x


def _static_rows_cached(case):
    """The cached rows of the packed static tensors."""
    rows, s = [], 0
    for r in _ints(case):
        n = r[0] + r[3]
        rows.append(torch.arange(s if case["mask"] == "beyond_alt" else s + r[0], s + n, device="cuda"))
        s += n
    return torch.cat(rows)


def _prepare_attn(case, seed):
    x = _attn_inputs(case, seed)
    st = {"case": case, "x": x, "groups": _groups(case), "scale": 1.0 / math.sqrt(case["dim"])}
    # the forward call's outputs
    st["o"] = torch.empty_like(x["q"])
    st["lse"] = torch.empty(x["q"].shape[:2], dtype=torch.float32, device="cuda")
    for qs, a, b in st["groups"]:
        keys, vals = _keys(x, a, b)
        for h in range(case["heads"]):
            s = (x["q"][qs, h].float() @ keys[h].t()) * st["scale"]
            lse = torch.logsumexp(s, 1)
            st["o"][qs, h] = (torch.exp(s - lse[:, None]) @ vals[h]).to(torch.bfloat16)
            st["lse"][qs, h] = lse
    st["grads"] = {n: torch.empty_like(x["q"]) for n in ("dq", "dk", "dv")}
    if case["kind"] == "step_bwd" and case["ref_grad"]:
        st["grads"].update(dk_ref=torch.empty_like(x["kc"]), dv_ref=torch.empty_like(x["vc"]))
    st["cached"] = _static_rows_cached(case) if case["kind"] == "build_bwd" else None
    if own:
        from paper_2608_21229_gb300 import refcache as rc

        st["rc"] = rc
        reqs = _ints(case)
        if case["kind"] == "full_bwd":
            st["cu"] = _cu([r[1] + r[2] + r[3] for r in reqs])
        else:
            seg = rc.Segments(case["heads"], case["dim"], _cu([r[1] + r[2] for r in reqs]), _cu([r[0] + r[3] for r in reqs]),
                              [r[0] for r in reqs], [r[1] for r in reqs])
            st["cache"] = rc.RefCache(seg, num_layers=1, mask_mode=case["mask"])
        if case["kind"] == "step_bwd":
            rows = _static_rows_cached(case)
            static = [torch.zeros(st["cache"].seg.static_rows, case["heads"], case["dim"], dtype=torch.bfloat16, device="cuda")
                      for _ in range(4)]
            static[1][rows], static[2][rows] = x["kc"], x["vc"]
            st["cache"].build(0, *static)
    return st


def _keys(x, a, b):
    """Keys and values [heads, keys, dim] in 32 bits: the call's own rows, then the cache's."""
    ks = [x["k"][a]] + ([x["kc"][b]] if _len(b) else [])
    vs = [x["v"][a]] + ([x["vc"][b]] if _len(b) else [])
    return _heads_first(torch.cat(ks)), _heads_first(torch.cat(vs))


def _positions(case):
    """Position (frame, y, x) of each row of the streams (all text rows, then all image rows), and its row in the packed requests."""
    text, image, text_rows, image_rows, at = [], [], [], [], 0
    for n, h, w, frames in _ints(case):
        i = torch.arange(n, device="cuda", dtype=torch.int32) + max(h, w) // 2
        text.append(i[:, None].expand(n, 3))
        f, y, x = (torch.arange(m, device="cuda", dtype=torch.int32) for m in (frames, h, w))
        image.append(torch.stack(torch.meshgrid(f, y - h // 2, x - w // 2, indexing="ij"), -1).reshape(-1, 3))
        text_rows.append(torch.arange(at, at + n, device="cuda", dtype=torch.int32))
        image_rows.append(torch.arange(at + n, at + n + frames * h * w, device="cuda", dtype=torch.int32))
        at += n + frames * h * w
    return torch.cat(text + image).contiguous(), torch.cat(text_rows + image_rows)


def _rope_inputs(case, seed):
    gen, h, d = _gen(seed), case["heads"], case["dim"]
    pos, rows = _positions(case)
    x = {"qkv": _randn(gen, (len(rows), 3, h, d), 1.5)}
    wd = torch.bfloat16 if case["wdtype"] == "bf16" else torch.float32
    if case["norm"]:
        x["wq"], x["wk"] = _randn(gen, (d,), 0.2, 1.0, wd), _randn(gen, (d,), 0.2, 1.0, wd)
    else:
        x["wq"] = x["wk"] = None
    if case["kind"] == "rope_bwd":
        for n in ("gq", "gk", "gv"):
            x[n] = _randn(gen, (len(rows), h, d))
    return x, pos, rows


def _prepare_rope(case, seed):
    x, pos, rows = _rope_inputs(case, seed)
    n, h, d = len(rows), case["heads"], case["dim"]
    st = {"case": case, "x": x, "pos": pos, "rows": rows}
    if case["kind"] == "rope_fwd":
        st["out"] = {k: torch.zeros(n, h, d, dtype=torch.bfloat16, device="cuda") for k in "qkv"}
    else:
        st["out"] = {"dqkv": torch.zeros_like(x["qkv"])}
        if case["norm"]:
            st["out"].update(dwq=torch.empty(d, dtype=torch.float32, device="cuda"), dwk=torch.empty(d, dtype=torch.float32, device="cuda"))
    if own:
        from paper_2608_21229_gb300 import refcache as rc

        st["rc"], st["rope"] = rc, rc.Rope(d, axes=AXES[d], theta=THETA, pairs=case["pairs"])
    else:
        # the rotation's frequencies and axes, which a program keeps with its model
        f = [THETA ** (-2.0 * j / a) for a in AXES[d] for j in range(a // 2)]
        st["freq"] = torch.tensor(f, dtype=torch.float64).to(torch.float32).cuda()
        st["axis"] = torch.tensor([i for i, a in enumerate(AXES[d]) for _ in range(a // 2)], device="cuda")
    return st


def _norm_inputs(case, seed):
    gen, c = _gen(seed), case["width"]
    lens = [int(n) for n in case["reqs"].split(";")]
    n, batch = sum(lens), len(lens)
    md = torch.bfloat16 if case["mods"] == "bf16" else torch.float32
    mods = _randn(gen, (batch, 6 * c), 0.3, 0.0, md)  # one projection's output: shift, scale and gate of both halves
    x = {"x": _randn(gen, (n, c), 2.0, 0.1), "branch": _randn(gen, (n, c), 1.0), "gate": mods[:, 2 * c:3 * c],
         "shift": mods[:, 3 * c:4 * c], "scale": mods[:, 4 * c:5 * c]}
    x["weight"] = _randn(gen, (c,), 0.2, 1.0, md) if case["weight"] else None
    x["post_weight"] = _randn(gen, (c,), 0.2, 1.0, md) if case["weight"] and case["post"] != "none" else None
    if case["kind"] == "norm_bwd":
        x["dy"], x["dx_out"] = _randn(gen, (n, c)), _randn(gen, (n, c))
    return x, lens


def _prepare_norm(case, seed):
    x, lens = _norm_inputs(case, seed)
    st = {"case": case, "x": x, "cu": _cu(lens)}
    n, c, batch = sum(lens), case["width"], len(lens)
    if case["kind"] == "norm_fwd":
        st["out"] = {"x_out": torch.empty_like(x["x"]), "y": torch.empty_like(x["x"])}
    else:
        st["out"] = {"dx": torch.empty_like(x["x"]), "d_branch": torch.empty_like(x["x"])}
        for k in ("d_gate", "d_scale", "d_shift"):
            st["out"][k] = torch.empty(batch, c, dtype=torch.float32, device="cuda")
        for k in ("weight", "post_weight"):
            if x[k] is not None:
                st["out"]["d_" + k] = torch.empty(c, dtype=torch.float32, device="cuda")
    if own:
        from paper_2608_21229_gb300 import refcache as rc

        st["rc"] = rc
    else:
        st["req"] = torch.repeat_interleave(torch.arange(batch, device="cuda"), torch.tensor(lens, device="cuda"))
        st["which"] = (torch.arange(batch, device="cuda")[:, None] == st["req"][None]).float()
    return st


def _clip_inputs(case, seed):
    gen, shapes = _gen(seed), _clip_shapes(case)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    flat = _randn(gen, (sum(math.prod(s) for s in shapes),), case["gain"], 0.0, dt)
    return flat, shapes


def _views(flat, shapes):
    return [t.view(s) for t, s in zip(flat.split([math.prod(s) for s in shapes]), shapes)]


def _prepare_clip(case, seed):
    flat, shapes = _clip_inputs(case, seed)
    out = torch.empty_like(flat, dtype=torch.float32 if case["out"] == "fp32" else flat.dtype)
    st = {"case": case, "grads": _views(flat, shapes), "out": out, "outs": _views(out, shapes),
          "norm": torch.empty((), dtype=torch.float32, device="cuda")}
    if own:
        from paper_2608_21229_gb300 import refcache as rc

        st["rc"] = rc
    return st


def prepare(case, seed):
    return {"attn": _prepare_attn, "rope": _prepare_rope, "norm": _prepare_norm, "clip": _prepare_clip}[case["op"]](case, seed)


# ---------------------------------------------------------------- one pass
def _run_attn(st):
    """dV = P^T dO, dP = dO V^T, dS = P (dP - sum(dO O)), dQ = scale dS K, dK = scale dS^T Q, with P = exp(scale Q K^T - lse)."""
    case, x, scale = st["case"], st["x"], st["scale"]
    sums = {n: torch.zeros(x["k"].shape, dtype=torch.float32, device="cuda") for n in ("dk", "dv")}
    if case["kind"] == "build_bwd" and case["ref_grad"]:
        sums["dk"][st["cached"]] += x["dk_ref"].float()
        sums["dv"][st["cached"]] += x["dv_ref"].float()
    g = st["grads"]
    for qs, a, b in st["groups"]:
        keys, vals = _keys(x, a, b)
        q, do = _heads_first(x["q"][qs]), _heads_first(x["do"][qs])
        delta = (do * _heads_first(st["o"][qs])).sum(-1, keepdim=True)
        p = torch.matmul(q, keys.transpose(1, 2)).mul_(scale).sub_(st["lse"][qs].t()[:, :, None]).exp_()
        dv = torch.matmul(p.transpose(1, 2), do)
        ds = torch.matmul(do, vals.transpose(1, 2)).sub_(delta).mul_(p).mul_(scale)
        del p
        dk = torch.matmul(ds.transpose(1, 2), q)
        g["dq"][qs] = torch.matmul(ds, keys).transpose(0, 1).to(torch.bfloat16)
        n = _len(a)
        sums["dk"][a] += dk[:, :n].transpose(0, 1)
        sums["dv"][a] += dv[:, :n].transpose(0, 1)
        if _len(b) and case["ref_grad"]:
            g["dk_ref"][b] = dk[:, n:].transpose(0, 1).to(torch.bfloat16)
            g["dv_ref"][b] = dv[:, n:].transpose(0, 1).to(torch.bfloat16)
    g["dk"].copy_(sums["dk"])
    g["dv"].copy_(sums["dv"])
    return g


def _run_attn_own(st):
    case, x, g = st["case"], st["x"], st["grads"]
    args = (x["q"], x["k"], x["v"], st["o"], st["lse"], x["do"], g["dq"], g["dk"], g["dv"])
    if case["kind"] == "full_bwd":
        st["rc"].full_attention_backward(st["cu"], *args)
    elif case["kind"] == "step_bwd":
        st["cache"].step_backward(0, *args, dk_ref=g.get("dk_ref"), dv_ref=g.get("dv_ref"))
    else:
        st["cache"].build_backward(0, *args, dk_ref=x.get("dk_ref"), dv_ref=x.get("dv_ref"))
    return g


def _pair_up(x, pairs):
    """x [..., dim] as its pairs' first and second members [..., dim / 2]."""
    return (x[..., 0::2], x[..., 1::2]) if pairs == "interleaved" else tuple(x.chunk(2, -1))


def _pair_down(a, b, pairs):
    return torch.stack((a, b), -1).flatten(-2) if pairs == "interleaved" else torch.cat((a, b), -1)


def _rotate(x, cos, sin, pairs):
    a, b = _pair_up(x, pairs)
    return _pair_down(a * cos - b * sin, a * sin + b * cos, pairs)


def _run_rope(st):
    """out[rows] = rotate(x / rms(x) * w, angle = position * frequency) of q and k, v moved; or the gradients of that."""
    case, x, pairs, rows = st["case"], st["x"], st["case"]["pairs"], st["rows"].long()
    angle = st["pos"].float()[:, st["axis"]] * st["freq"]
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    out = st["out"]
    if case["kind"] == "rope_fwd":
        for i, (n, w) in enumerate((("q", x["wq"]), ("k", x["wk"]))):
            t = x["qkv"][:, i].float()
            if case["norm"]:
                t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * w.float()
            out[n][rows] = _rotate(t, cos, sin, pairs).to(torch.bfloat16)
        out["v"][rows] = x["qkv"][:, 2]
        return out
    for i, (n, w) in enumerate((("gq", x["wq"]), ("gk", x["wk"]))):
        g = _rotate(x[n][rows].float(), cos, -sin, pairs)
        if case["norm"]:
            t = x["qkv"][:, i].float()
            r = torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS)
            gw = g * w.float()
            out["dwq" if i == 0 else "dwk"].copy_((g * t * r).sum((0, 1)))
            g = r * gw - t * (r ** 3 * (t * gw).mean(-1, keepdim=True))
        out["dqkv"][:, i] = g.to(torch.bfloat16)
    out["dqkv"][:, 2] = x["gv"][rows]
    return out


def _run_rope_own(st):
    rc, case, x, out = st["rc"], st["case"], st["x"], st["out"]
    q, k, v = x["qkv"].unbind(1)
    if case["kind"] == "rope_fwd":
        rc.qkv_rope(st["rope"], st["pos"], q, k, v, out["q"], out["k"], out["v"], x["wq"], x["wk"], rows=st["rows"], eps=EPS)
    else:
        rc.qkv_rope_backward(st["rope"], st["pos"], q, k, x["gq"], x["gk"], x["gv"], *out["dqkv"].unbind(1), x["wq"], x["wk"],
                             out.get("dwq"), out.get("dwk"), rows=st["rows"], eps=EPS)
    return out


def _normed(x, kind):
    """The norm of rows of x, and the factor 1 / deviation."""
    c = x - x.mean(-1, keepdim=True) if kind == "layer" else x
    r = torch.rsqrt(c.square().mean(-1, keepdim=True) + EPS)
    return c * r, r


def _normed_grad(g, xhat, r, kind):
    d = g - xhat * (g * xhat).mean(-1, keepdim=True)
    return r * (d - g.mean(-1, keepdim=True)) if kind == "layer" else r * d


def _run_norm(st):
    """x_out = x + gate h, h = the branch or its norm; y = norm(x_out) weight (1 + scale) + shift; or the gradients of that."""
    case, x, req, out = st["case"], st["x"], st["req"], st["out"]
    gate, scale, shift = (x[n].float()[req] for n in ("gate", "scale", "shift"))
    one = torch.ones(case["width"], device="cuda")
    w = one if x["weight"] is None else x["weight"].float()
    pw = one if x["post_weight"] is None else x["post_weight"].float()
    f = x["branch"].float()
    fhat, fr = _normed(f, case["post"]) if case["post"] != "none" else (f, None)
    h = fhat * pw
    if case["kind"] == "norm_fwd":
        t = x["x"].float() + gate * h
        out["x_out"].copy_(t)
        out["y"].copy_(_normed(t, case["norm"])[0] * w * (1 + scale) + shift)
        return out
    dy = x["dy"].float()
    xhat, r = _normed(x["x"].float(), case["norm"])  # x is the stream after the branch was added
    d = x["dx_out"].float() + _normed_grad(dy * (1 + scale) * w, xhat, r, case["norm"])
    dh = gate * d
    out["dx"].copy_(d)
    out["d_branch"].copy_(_normed_grad(dh * pw, fhat, fr, case["post"]) if case["post"] != "none" else dh)
    out["d_gate"].copy_(st["which"] @ (d * h))
    out["d_scale"].copy_(st["which"] @ (dy * xhat * w))
    out["d_shift"].copy_(st["which"] @ dy)
    if "d_weight" in out:
        out["d_weight"].copy_((dy * (1 + scale) * xhat).sum(0))
    if "d_post_weight" in out:
        out["d_post_weight"].copy_((dh * fhat).sum(0))
    return out


def _run_norm_own(st):
    rc, case, x, out = st["rc"], st["case"], st["x"], st["out"]
    how = {"norm": case["norm"], "post_norm": None if case["post"] == "none" else case["post"], "eps": EPS}
    if case["kind"] == "norm_fwd":
        rc.gated_norm(st["cu"], x["x"], out["y"], branch=x["branch"], x_out=out["x_out"], gate=x["gate"], scale=x["scale"],
                      shift=x["shift"], weight=x["weight"], post_weight=x["post_weight"], **how)
    else:
        rc.gated_norm_backward(st["cu"], x["x"], x["dy"], out["dx"], branch=x["branch"], dx_out=x["dx_out"], d_branch=out["d_branch"],
                               gate=x["gate"], scale=x["scale"], weight=x["weight"], post_weight=x["post_weight"],
                               d_gate=out["d_gate"], d_scale=out["d_scale"], d_shift=out["d_shift"], d_weight=out.get("d_weight"),
                               d_post_weight=out.get("d_post_weight"), **how)
    return out


def _run_clip(st):
    norm = torch.stack([g.float().square().sum() for g in st["grads"]]).sum().sqrt()
    coef = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    for g, o in zip(st["grads"], st["outs"]):
        o.copy_(g.float() * coef)
    st["norm"].copy_(norm)
    return {"norm": st["norm"], "grads": st["out"]}


def _run_clip_own(st):
    st["rc"].clip_gradients(st["grads"], MAX_NORM, out=st["outs"], norm=st["norm"])
    return {"norm": st["norm"], "grads": st["out"]}


def run(st):
    op = st["case"]["op"]
    if own:
        return {"attn": _run_attn_own, "rope": _run_rope_own, "norm": _run_norm_own, "clip": _run_clip_own}[op](st)
    return {"attn": _run_attn, "rope": _run_rope, "norm": _run_norm, "clip": _run_clip}[op](st)


# ---------------------------------------------------------------- the same in 64 bits
def _exact_attn(case, seed):
    """Gradients of softmax attention from its own probabilities, head by head (q, k, v and the output's gradient alone)."""
    if work(case)["flops"] > 5e12:
        return None
    x, scale = _attn_inputs(case, seed), 1.0 / math.sqrt(case["dim"])
    z = lambda t: torch.zeros(t.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out = {"dq": z(x["q"]), "dk": z(x["k"]), "dv": z(x["v"])}
    if case["kind"] == "step_bwd" and case["ref_grad"]:
        out.update(dk_ref=z(x["kc"]), dv_ref=z(x["vc"]))
    for qs, a, b in _groups(case):
        for h in range(case["heads"]):
            k, v = x["k"][a, h].double(), x["v"][a, h].double()
            if _len(b):
                k, v = torch.cat((k, x["kc"][b, h].double())), torch.cat((v, x["vc"][b, h].double()))
            for r in range(qs.start, qs.stop, 2048):
                rows = slice(r, min(r + 2048, qs.stop))
                q, do = x["q"][rows, h].double(), x["do"][rows, h].double()
                p = torch.softmax(q @ k.T * scale, 1)
                dp = do @ v.T
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * scale
                out["dq"][rows, h] = ds @ k
                dk, dv = ds.T @ q, p.T @ do
                out["dk"][a, h] += dk[:_len(a)]
                out["dv"][a, h] += dv[:_len(a)]
                if "dk_ref" in out and _len(b):
                    out["dk_ref"][b, h] += dk[_len(a):]
                    out["dv_ref"][b, h] += dv[_len(a):]
    if case["kind"] == "build_bwd" and case["ref_grad"]:
        rows = _static_rows_cached(case)
        out["dk"][rows] += x["dk_ref"].double()
        out["dv"][rows] += x["dv_ref"].double()
    return out


def _exact_rope(case, seed):
    """The rotation as a product of complex numbers; the gradients by torch's differentiation of the 64-bit definition."""
    x, pos, rows = _rope_inputs(case, seed)
    d, rows = case["dim"], rows.long()
    freq = torch.cat([torch.pow(torch.tensor(THETA, dtype=torch.float64), -torch.arange(0, a, 2, dtype=torch.float64) / a) for a in AXES[d]]).cuda()
    angle = torch.cat([pos[:, i:i + 1].double().expand(-1, a // 2) for i, a in enumerate(AXES[d])], 1) * freq
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def of(t, w):
        if w is not None:
            t = t / (t.square().mean(-1, keepdim=True) + EPS).sqrt() * w
        if case["pairs"] == "interleaved":
            return torch.view_as_real(torch.view_as_complex(t.reshape(*t.shape[:-1], d // 2, 2).contiguous()) * turn).flatten(-2)
        c = torch.complex(t[..., :d // 2].contiguous(), t[..., d // 2:].contiguous()) * turn
        return torch.cat((c.real, c.imag), -1)

    out = {}
    if case["kind"] == "rope_fwd":
        for i, (n, w) in enumerate((("q", x["wq"]), ("k", x["wk"]))):
            out[n] = torch.zeros(len(rows), case["heads"], d, dtype=torch.float64, device="cuda")
            out[n][rows] = of(x["qkv"][:, i].double(), None if w is None else w.double())
        out["v"] = torch.zeros_like(out["q"])
        out["v"][rows] = x["qkv"][:, 2].double()
        return out
    out["dqkv"] = torch.zeros(x["qkv"].shape, dtype=torch.float64, device="cuda")
    for i, (n, w) in enumerate((("q", x["wq"]), ("k", x["wk"]))):
        t = x["qkv"][:, i].double().requires_grad_()
        w = None if w is None else w.double().requires_grad_()
        got = torch.autograd.grad(of(t, w), (t,) if w is None else (t, w), x["g" + n][rows].double())
        out["dqkv"][:, i] = got[0]
        if w is not None:
            out["dw" + n] = got[1]
    out["dqkv"][:, 2] = x["gv"][rows].double()
    return out


def _exact_norm(case, seed):
    """Request by request; the gradients by torch's differentiation of the 64-bit definition."""
    x, lens = _norm_inputs(case, seed)
    c = case["width"]

    def norm(t, kind):
        if kind == "layer":
            return (t - t.mean(-1, keepdim=True)) / (t.var(-1, unbiased=False, keepdim=True) + EPS).sqrt()
        return t / (t.square().mean(-1, keepdim=True) + EPS).sqrt() if kind == "rms" else t

    x = {k: None if v is None else v.double() for k, v in x.items()}
    out, at = {}, 0
    w = torch.ones(c, dtype=torch.float64, device="cuda") if x["weight"] is None else x["weight"]
    pw = torch.ones(c, dtype=torch.float64, device="cuda") if x["post_weight"] is None else x["post_weight"]
    for i, n in enumerate(lens):
        rows = slice(at, at + n)
        at += n
        gate, scale, shift = x["gate"][i], x["scale"][i], x["shift"][i]
        if case["kind"] == "norm_fwd":
            t = x["x"][rows] + gate * (norm(x["branch"][rows], case["post"]) * pw)
            got = {"x_out": t, "y": norm(t, case["norm"]) * w * (1 + scale) + shift}
            for k, v in got.items():
                out.setdefault(k, []).append(v)
            continue
        # the stream as a sum of its value and of terms that are zero here, for their gradients
        leaf = {k: v.clone().requires_grad_() for k, v in (("dx", x["x"][rows]), ("d_branch", x["branch"][rows]), ("d_gate", gate),
                                                         ("d_scale", scale), ("d_shift", shift), ("d_weight", w), ("d_post_weight", pw))}
        h = norm(leaf["d_branch"], case["post"]) * leaf["d_post_weight"]
        add = leaf["d_gate"] * h
        t = leaf["dx"] + (add - add.detach())
        y = norm(t, case["norm"]) * leaf["d_weight"] * (1 + leaf["d_scale"]) + leaf["d_shift"]
        got = torch.autograd.grad((y, t), list(leaf.values()), (x["dy"][rows], x["dx_out"][rows]))
        for k, v in zip(leaf, got):
            out.setdefault(k, []).append(v)
    if case["kind"] == "norm_fwd":
        return {k: torch.cat(v) for k, v in out.items()}
    got = {k: torch.cat(out[k]) for k in ("dx", "d_branch")}
    got.update({k: torch.stack(out[k]) for k in ("d_gate", "d_scale", "d_shift")})
    if x["weight"] is not None:
        got["d_weight"] = sum(out["d_weight"])
    if x["post_weight"] is not None:
        got["d_post_weight"] = sum(out["d_post_weight"])
    return got


def _exact_clip(case, seed):
    flat, _ = _clip_inputs(case, seed)
    norm = torch.linalg.vector_norm(flat, dtype=torch.float64)
    return {"norm": norm, "grads": flat.double() * min(1.0, MAX_NORM / (float(norm) + 1e-6))}


def exact(case, seed):
    return {"attn": _exact_attn, "rope": _exact_rope, "norm": _exact_norm, "clip": _exact_clip}[case["op"]](case, seed)
