"""Counts that no launch takes: the whole list is looked at before its first tensor is."""
import pytest

from test_host_create import run_child  # noqa: F401  (a fixture)


@pytest.mark.parametrize("count", [1 << 46, 1 << 62, (1 << 63) - 1, (1 << 63) - 16384])
@pytest.mark.parametrize("first", [0, 1, 600])
def test_a_list_of_too_many_elements_launches_nothing(run_child, count, first):  # noqa: F811
    """`first` tensors of one element before it, which may fill a launch of their own."""
    out = run_child(f"""
n = {first} + 2
P = 1 << 20
a = (ctypes.c_void_p * n)(*[P] * n), None, (ctypes.c_int64 * n)(*[1] * {first}, {count}, 1), (ctypes.c_int32 * n)(*[0] * n)
code = L.refcache_clip_gradients(n, *a, 1.0, None, P, None)
print(json.dumps([code, rc.last_error(), cudart.host_cudart_launches()]))""")
    assert out[0] == -1 and "too many elements" in out[1] and out[2] == 0, out


def test_the_largest_list_that_a_launch_takes(run_child):  # noqa: F811
    out = run_child("""
P, n = 1 << 20, 2
a = (ctypes.c_void_p * n)(*[P] * n), None, (ctypes.c_int64 * n)(((1 << 31) - 4) << 14, 5), (ctypes.c_int32 * n)(*[0] * n)
code = L.refcache_clip_gradients(n, *a, 1.0, None, P, None)
print(json.dumps([code, cudart.host_cudart_launches()]))""")
    assert out == [0, 2]
