"""Properties of the 8-bit products' source that no run shows: what only matters after a wait has run out."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_21229_gb300", "csrc")


def _code(name):
    return re.sub(r"\s+", " ", re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read()))


def test_tensor_memory_is_freed_behind_every_mma_that_was_issued():
    """The sums' warps may give up while the MMAs they wait for go on: the warp that issued them waits for them
    itself, whether or not its own waits were fulfilled, before tensor memory is freed."""
    few = _code("f8_few.cuh")
    loop, freed = few.index("mx_mma(tmem"), few.index("tcgen05.dealloc")
    own = few.index("if (elect_one()) { if (issued) commit(bar(L::kAccFull)); if (issued || sums > 0) drain(bar(L::kAccFull), static_cast<uint32_t>(issued ? sums : sums - 1) & 1u")
    assert loop < own < freed
    pair = _code("f8_pair.cuh")
    finish = pair[pair.index("void finish_mmas("):]
    assert "if (issued && elect_one()) { tc2_commit_mc(bar(L::kDone), 1); drain(bar(L::kDone), 0u" in finish[:300]
    for name in ("f8_linear.cuh", "f8_wgrad.cuh"):
        code = _code(name)
        assert code.index("issued = true") < code.index("c.finish_mmas(issued)") < code.index("c.leave(")
