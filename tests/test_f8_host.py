"""The host side of the 8-bit linear layers without a GPU: the CUDA runtime's calls go to stand-ins, in a child process."""
import json
import os
import subprocess
import sys

import pytest

from paper_2608_21229_gb300 import build as cbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import ctypes, json, sys
sys.path.insert(0, {root!r})
from paper_2608_21229_gb300 import refcache as rc
cudart = ctypes.CDLL(None)
L = rc.load()
P = 0x1000000
rows = lambda i, n, w: ctypes.byref(rc._F8Rows(n, w, P * i, P * (i + 1), P * (i + 2)))
weight = lambda i, n, k: ctypes.byref(rc._F8Weight(n, k, *(P * (i + j) for j in range(6))))
CALLS = dict(
    linear=lambda: L.refcache_f8_linear(rows(1, 600, 1024), weight(4, 512, 1024), 0, None, 0, P * 10, 512, None),
    gelu=lambda: L.refcache_f8_linear_gelu(rows(1, 600, 1024), weight(4, 512, 1024), None, 0, 0, rows(10, 600, 512), None, None),
    wgrad=lambda: L.refcache_f8_weight_grad(P * 1, 512, rows(2, 600, 1024), 512, None, P * 5, 1, None, P * 10, None))


def call(name):
    before = cudart.host_cudart_launches()
    code = CALLS[name]()
    return [code, cudart.host_cudart_launches() - before, rc.last_error() if code else ""]


{body}
"""


@pytest.fixture(scope="module")
def run_child(tmp_path_factory):
    where = tmp_path_factory.mktemp("cudart")
    shims = []
    for name in ("host_clusters", "host_cudart"):
        shims.append(str(where / f"{name}.so"))
        subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", shims[-1], os.path.join(ROOT, "tests", "c", f"{name}.c")], check=True)
    cbuild.build()

    def run(body):
        r = subprocess.run([sys.executable, "-c", CHILD.format(root=ROOT, body=body)], capture_output=True, text=True,
                           timeout=300, env=dict(os.environ, LD_PRELOAD=":".join(shims)))
        assert r.returncode == 0, r.stderr
        return json.loads(r.stdout.splitlines()[-1])

    return run


@pytest.mark.parametrize("name", ["linear", "gelu", "wgrad"])
def test_a_count_of_clusters_that_fails_is_reported_before_anything_is_launched(run_child, name):
    """Not answered by a guess that is kept for the process, nor by an error that the runtime reports behind a launch: the
    call fails, and the next one finds the runtime without an error and asks again."""
    failed, none, good, again = run_child(f"""
out = []
for fail, none in ((1, 0), (0, 1), (0, 0), (1, 0)):
    cudart.host_clusters_set(fail, none)
    out.append(call({name!r}))
print(json.dumps(out))""")
    assert failed[0] == -4 and failed[1] == 0 and "cudaOccupancyMaxActiveClusters" in failed[2]
    assert none[0] == -4 and none[1] == 0 and none[2]
    assert good[0] == 0 and good[1] >= 1
    assert again == good  # (counted once)
