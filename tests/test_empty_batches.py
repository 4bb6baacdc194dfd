"""Batches without rows: torch gives the address NULL for a tensor without elements, so nothing is missing there."""
import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

from test_host_create import run_child  # noqa: F401  (a fixture)

BF16 = torch.bfloat16


def test_gated_norm_without_rows_needs_no_tensors(run_child):  # noqa: F811
    """Through the C entries, on host-memory stand-ins for the runtime: forward launches nothing, the gradient only the
    sums over no rows; with rows the tensors are still asked for."""
    out = run_child("""
P = 1 << 20
def go(cu, branch, dy, dx_out, sums):
    arr = (ctypes.c_int32 * len(cu))(*cu)
    c = rc._GatedNorm(batch=len(cu) - 1, width=64, cu_rows=arr, norm=1, post_norm=2, mod_f32=0, eps=1e-6, weight=P, post_weight=P)
    n = cudart.host_cudart_launches()
    fwd = L.refcache_gated_norm(ctypes.byref(c), P, branch, P, P, None)
    mid = cudart.host_cudart_launches()
    bwd = L.refcache_gated_norm_backward(ctypes.byref(c), P, branch, dy, dx_out, P, branch and P, *sums, P, None)
    return fwd, mid - n, bwd, cudart.host_cudart_launches() - mid
every, none = [P] * 5, [None] * 5
print(json.dumps([go((0, 0, 0), None, None, None, every), go((0, 0), P, None, None, none), go((0, 2), None, P, None, every),
                  go((0, 2), P, None, None, none), go((0, 2), P, P, None, every)]))""")
    assert out[0] == [0, 0, 0, 1] and out[1] == [0, 0, 0, 0]
    assert out[2][:2] == [-1, 0] and out[2][2:] == [-1, 0]  # no branch for x_out, d_gate and d_post_weight
    assert out[3][:2] == [0, 1] and out[3][2:] == [-1, 0]  # neither dy nor dx_out
    assert out[4] == [0, 1, 0, 2]


@pytest.mark.gpu
@pytest.mark.parametrize("branch", [False, True])
@pytest.mark.parametrize("B", [1, 3, 70])
def test_gated_norm_of_an_empty_batch(branch, B):
    cu, W = [0] * (B + 1), 512
    row = lambda: torch.empty(0, W, dtype=BF16, device="cuda")  # noqa: E731
    f32 = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    mod = torch.ones(B, W, dtype=BF16, device="cuda")
    w = torch.ones(W, dtype=BF16, device="cuda")
    part = dict(branch=row(), gate=mod, post_weight=w, post_norm="rms") if branch else {}
    rcb.gated_norm(cu, row(), row(), x_out=row() if branch else None, scale=mod, shift=mod, weight=w, **part)
    got = dict(d_scale=f32(B, W), d_shift=f32(B, W), d_weight=f32(W))
    if branch:
        got.update(d_gate=f32(B, W), d_post_weight=f32(W))
    for dx_out in (None, row()):
        for t in got.values():
            t.fill_(float("nan"))
        rcb.gated_norm_backward(cu, row(), row(), row(), dx_out=dx_out, d_branch=row() if branch else None, scale=mod, weight=w, **part, **got)
        assert all((t == 0).all() for t in got.values())
    with pytest.raises(rcb.RefCacheError, match="without a branch"):  # (of rows there are some)
        x = torch.zeros(B, W, dtype=BF16, device="cuda")
        rcb.gated_norm_backward(list(range(B + 1)), x, x, x.clone(), d_gate=f32(B, W))


@pytest.mark.gpu
def test_the_other_operators_of_an_empty_batch():
    H, D = 2, 64
    thd = lambda: torch.empty(0, H, D, dtype=BF16, device="cuda")  # noqa: E731
    rope, pos, w = rcb.Rope(D, (8, 28, 28)), torch.empty(0, 3, dtype=torch.int32, device="cuda"), torch.ones(D, device="cuda")
    rcb.qkv_rope(rope, pos, thd(), thd(), thd(), thd(), thd(), thd(), w, w)
    dw = [torch.full((D,), float("nan"), device="cuda") for _ in range(2)]
    rcb.qkv_rope_backward(rope, pos, thd(), thd(), thd(), thd(), thd(), thd(), thd(), thd(), w, w, *dw)
    assert all((t == 0).all() for t in dw)
    lse = torch.empty(0, H, device="cuda")
    rcb.full_attention_backward([0, 0, 0], thd(), thd(), thd(), thd(), lse, thd(), thd(), thd(), thd())
    assert rcb.clip_gradients([thd(), lse], 1.0).item() == 0.0
    assert rcb.status() == rcb.OK
