"""Tensors on another device than the one a call runs on are refused before anything is launched: the kernels would
read them without a mapping, or without order.  On stand-ins for tensors and for the library, which need no GPU."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
H, D, N, W = 2, 64, 6, 128


class T:
    """What the binding asks of a tensor."""

    def __init__(self, shape, dtype=BF16, device=0):
        self.shape, self.dtype, self.at = torch.Size(shape), dtype, device
        self.device = torch.device("cpu") if device < 0 else torch.device("cuda", device)
        self.is_cuda = device >= 0

    def get_device(self):
        return self.at

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x1000

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self):
        return tuple(torch.Size(self.shape[i + 1:]).numel() for i in range(len(self.shape)))


class Lib:
    """Records calls in place of making them."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(self.real, name)
        return lambda *a: self.calls.append(name) or 0


def thd(n=N):
    return (n, H, D)


def calls():
    """name -> (the call on tensors by name, the tensors)."""
    rope = rcb.Rope(D, (8, 28, 28))
    seg = rcb.Segments(H, D, [0, N], [0, N], [0])
    cache = rcb.RefCache.__new__(rcb.RefCache)
    cache.seg, cache.num_layers, cache.mask_mode, cache.h, cache.mem = seg, 1, "beyond", None, T((1,), torch.uint8)
    attn = {n: T(thd()) for n in ("q", "k", "v", "o")}
    grads = {**attn, "lse": T((N, H), F32), **{n: T(thd()) for n in ("d_o", "dq", "dk", "dv")}}
    refs = {n: T(thd()) for n in ("dk_ref", "dv_ref")}
    w = {"weight_q": T((D,)), "weight_k": T((D,))}
    pos = {"positions": T((N, 3), I32), "rows": T((N,), I32)}
    rows = lambda *names: {n: T((N, W)) for n in names}  # noqa: E731
    mods = lambda *names: {n: T((2, W), F32) for n in names}  # noqa: E731
    vecs = lambda *names: {n: T((W,), F32) for n in names}  # noqa: E731
    cu = [0, 2, N]
    return {
        "full_attention": (lambda t: rcb.full_attention([0, N], **t), {**attn, "lse": T((N, H), F32)}),
        "full_attention_noalloc": (lambda t: rcb.full_attention_noalloc([0, N], **t), {**attn, "lse": T((N, H), F32)}),
        "build": (lambda t: cache.build(0, **t), {**attn, "lse": T((N, H), F32)}),
        "step": (lambda t: cache.step(0, **t), {**attn, "lse": T((N, H), F32)}),
        "full_attention_backward": (lambda t: rcb.full_attention_backward([0, N], **t), grads),
        "step_backward": (lambda t: cache.step_backward(0, **t), {**grads, **refs}),
        "build_backward": (lambda t: cache.build_backward(0, **t), {**grads, **refs}),
        "qkv_rope": (lambda t: rcb.qkv_rope(rope, **t), {**pos, **{n: T(thd()) for n in ("q", "k", "v", "q_out", "k_out", "v_out")}, **w}),
        "qkv_rope_backward": (lambda t: rcb.qkv_rope_backward(rope, **t), {
            **pos, **{n: T(thd()) for n in ("q", "k", "dq_out", "dk_out", "dv_out", "dq", "dk", "dv")}, **w,
            "dweight_q": T((D,), F32), "dweight_k": T((D,), F32)}),
        "gated_norm": (lambda t: rcb.gated_norm(cu, post_norm="rms", **t), {
            **rows("x", "y", "branch", "x_out"), **mods("gate", "scale", "shift"), **vecs("weight", "post_weight")}),
        "gated_norm_backward": (lambda t: rcb.gated_norm_backward(cu, post_norm="rms", **t), {
            **rows("x_out", "dy", "dx", "branch", "dx_out", "d_branch"), **mods("gate", "scale", "d_gate", "d_scale", "d_shift"),
            **vecs("weight", "post_weight", "d_weight", "d_post_weight")}),
        "clip_gradients": (lambda t: rcb.clip_gradients([t["a"], t["b"]], 1.0, out=[t["a_out"], t["b_out"]], norm=t["norm"]), {
            "a": T((5, 7)), "b": T((9,), F32), "a_out": T((35,)), "b_out": T((9,)), "norm": T((), F32)}),
    }


@pytest.fixture
def lib(monkeypatch):
    from paper_2608_21229_gb300 import build as cbuild

    cbuild.build()
    real = rcb.load()
    made = calls()  # (Rope asks the library)
    fake = Lib(real)
    monkeypatch.setattr(rcb, "load", lambda path=None: fake)
    monkeypatch.setattr(rcb, "_get_device", lambda: 0, raising=False)
    monkeypatch.setattr(rcb, "_stream", lambda s: 0)
    monkeypatch.setattr(rcb, "_work", lambda nbytes, like, stream: T((nbytes,), torch.uint8, like.get_device()))
    return fake, made


NAMES = ["full_attention", "full_attention_noalloc", "build", "step", "full_attention_backward", "step_backward", "build_backward", "qkv_rope",
         "qkv_rope_backward", "gated_norm", "gated_norm_backward", "clip_gradients"]


@pytest.mark.parametrize("name", NAMES)
def test_every_tensor_is_on_the_calls_device(lib, name):
    fake, made = lib
    go, tensors = made[name]
    go(tensors)
    assert len(fake.calls) == 1
    for bad in tensors:
        for device, match in ((1, "cuda:1, the call runs on cuda:0"), (-1, "must live on the GPU")):
            t = {n: T(x.shape, x.dtype, device if n == bad else 0) for n, x in tensors.items()}
            with pytest.raises(ValueError, match=match):
                go(t)
    if name not in ("build", "step", "step_backward", "build_backward"):  # (the library refuses a cache of another device)
        with pytest.raises(ValueError, match="cuda:1"):
            go({n: T(x.shape, x.dtype, 1) for n, x in tensors.items()})
    assert len(fake.calls) == 1
