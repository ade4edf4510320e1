"""Waits of the matrix product that are checked by reading its source: a
warp that gives up a bounded wait leaves its loop, so a barrier inside the loop
that counts on it would be a wait without a limit."""

import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_02805_gb300", "csrc",
                      "gemm.cuh")


def _code():
    return re.sub(r"//[^\n]*", "", open(SOURCE).read())


def test_no_plain_barrier_among_the_epilogue_warps():
    """Barrier 1 counts the epilogue warps. It carries whether one of them gave up, and every way out of the loop over
    tiles goes through it."""
    code = _code()
    assert not re.search(r"bar(?:rier)?(?:\.cta)?\.(?:sync|arrive)\s+1\b", code)
    assert len(re.findall(r"bar\.red\.or\.pred q, 1,", code)) == 1
    start = code.index("for (int i = 0; another;)")
    epilogue = code[start:code.index("if (!ok && lane == 0) atomicExch", start)]
    # before an accumulator's values are used: the warps that could not get them say so and leave
    assert re.search(r"if \(!ok\) \{\s*if constexpr \(EPI == kEpiStats\) epilogue_sync\(true\);\s*break;\s*\}", epilogue)
    # where the quarters of a row meet: all leave with the one that gave up
    assert re.search(r"if \(!\(ok = !epilogue_sync\(false\)\)\) break;", epilogue)
    assert len(re.findall(r"epilogue_sync\(", epilogue)) == 2


def test_polling_is_bounded():
    """No loop around a poll without a limit, and no wait outside umma::bar_wait."""
    code = _code()
    assert "try_wait" not in code and "test_wait" not in code
    assert not re.search(r"while\s*\(\s*(?:true|1|!)", code) and not re.search(r"for\s*\(\s*;\s*;", code)
