"""The keys kernel of the attention's gradients starts while the queries kernel before it runs: what orders its
reads behind the kernels before both."""
import ctypes
import os
import re

import pytest
import torch

from paper_2608_21229_gb300 import refcache as rcb

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_21229_gb300", "csrc")


def _code(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_a_cta_starts_behind_a_wait_or_an_acquired_ticket():
    """griddepcontrol.wait alone promises that earlier writes are visible.  A CTA that goes on without it has
    acquired what the queries kernel released behind its own wait, for all its threads and for its TMA loads."""
    code, ptx = _code("attn_bwd_tc.cuh"), _code("ptx.cuh")
    enter = code[code.index("bool enter("):]
    enter = re.sub(r"\s+", " ", enter[:enter.index("return true;")])
    taken = enter.index("const bool passed = __syncthreads_or(late && threadIdx.x == 0 && ld_acquire_gpu(a.passed) == a.ticket)")
    go = enter.index("if (passed) fence_proxy_async_global(); else grid_dependency_wait();")
    given = enter.index("if (says && blockIdx.x == 0) st_release_gpu(a.passed, a.ticket); grid_launch_dependents();")
    assert taken < go < given
    for op in ("st.release.gpu.global.u64", "ld.acquire.gpu.global.u64", "fence.proxy.async.global"):
        assert op in ptx, op
    # the queries kernel says it, the keys kernel behind it looks for it, waits at its end and sets the word back
    assert "enter(c, smem_raw, args, maps, true, false)" in code and "enter(c, smem_raw, args, maps, false, args.behind_queries != 0)" in code
    keys = re.sub(r"\s+", " ", code[code.index("attn_bwd_keys_kernel("):code.index("attn_bwd_queries_kernel(")])
    assert "if (args.behind_queries) { grid_dependency_wait(); if (blockIdx.x == 0 && threadIdx.x == 0) st_release_gpu(args.passed, 0); }" in keys


def _call(work, n, H, D, t, out, lse):
    cu = (ctypes.c_int32 * 2)(0, n)
    ptrs = [x.data_ptr() for x in (t[0], t[1], t[2], t[3], lse, t[4], *out, work)]
    code = rcb.load().full_attention_backward(1, H, D, cu, *ptrs, D ** -0.5, rcb._stream(None))
    assert code == rcb.OK, rcb.last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("H,D,n", [(2, 64, 300), (24, 128, 900)])
def test_replays_follow_their_inputs(H, D, n):
    """Inputs written by the kernel right before, over one workspace that held something else: every replay of a graph
    gives the bits of a call that nothing overlaps."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    sets = []
    for _ in range(3):
        q, k, v, do = (torch.randn(n, H, D, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(4))
        o, lse = torch.empty_like(q), torch.empty(n, H, device="cuda")
        rcb.full_attention([0, n], q, k, v, o, lse)
        sets.append((torch.stack((q, k, v, o, do)), lse))
    nbytes = rcb.load().refcache_backward_bytes(n, H)
    want = []
    for t, lse in sets:
        out = torch.full((3, n, H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        _call(torch.full((nbytes,), 0xFF, dtype=torch.uint8, device="cuda"), n, H, D, t, out, lse)
        torch.cuda.synchronize()
        want.append(out)
    t, lse, source, source_lse = (torch.empty_like(sets[0][i]) for i in (0, 1, 0, 1))
    out = torch.empty_like(want[0])
    work = torch.randint(0, 256, (nbytes,), dtype=torch.uint8, device="cuda", generator=gen)

    def calls():
        t.copy_(source)
        lse.copy_(source_lse)
        _call(work, n, H, D, t, out, lse)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(30):
        x, y = sets[i % 3]
        source.copy_(x)
        source_lse.copy_(y)
        out.fill_(7.0)
        (graph.replay if i % 4 else calls)()
        assert torch.equal(out, want[i % 3]), i
    assert rcb.status() == rcb.OK
