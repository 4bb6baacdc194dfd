"""The limit of the kernels' waits."""
from paper_2608_21229_gb300 import build as cbuild
from paper_2608_21229_gb300 import refcache as rcb

LEAST = 1_000_000


def test_the_limit_leaves_time_for_what_is_in_flight():
    """A kernel that gives up waits no longer than the limit for its own loads and MMAs: shorter limits than they
    can take count as a millisecond."""
    cbuild.build()
    old = rcb.set_wait_timeout_ns(50_000_000)
    try:
        for asked, kept in ((0, LEAST), (1, LEAST), (LEAST - 1, LEAST), (LEAST, LEAST), (LEAST + 1, LEAST + 1), (1 << 63, 1 << 63)):
            rcb.set_wait_timeout_ns(asked)
            assert rcb.set_wait_timeout_ns(50_000_000) == kept
    finally:
        rcb.set_wait_timeout_ns(old)
