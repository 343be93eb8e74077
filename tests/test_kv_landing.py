"""Copies and products that are under way land before a CTA of the paged attention kernels
ends or frees tensor memory, whichever of its roles gives up a wait, and when.  A wait that
gives up cannot be brought about on a healthy GPU: the sources are read.  No GPU."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_02474_gb300", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def body(text, head):
    """The braces that follow `head`."""
    at = text.index("{", text.index(head))
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i + 1]


def test_the_wait_for_landing_is_bounded_and_asks_nobody():
    wait = body(source("common.cuh"), "mbar_land(")
    assert "limit_ns" in wait and "abort" not in wait


@pytest.mark.parametrize("name,roles", [
    ("kv_decode.cu", {"if (warp == C::WARPS) {": ["full"]}),
    ("kv_chunk.cu", {"if (warp == 3) {": ["q_full"], "else if (warp == 0) {": ["raw_full", "k_first", "pair"],
                     "else if (warp == 1) {": ["drain"]}),
])
def test_every_role_waits_for_what_it_began(name, roles):
    text = source(name)
    assert "if (*abort_v" not in text                  # roles give up after another one has looked
    for role, barriers in roles.items():
        part = body(text, role)
        for bar in barriers:
            assert re.search(r"mbar_land\(&(sh\.)?%s\b" % bar, part), (role, bar)
            assert not re.search(r"mbar_wait\(&(sh\.)?%s\b[^;]*nullptr" % bar, part), (role, bar)


def test_the_pairs_that_the_chunk_kernel_waits_for():
    """Copy li of K_0 V_0 K_1 V_1 .. belongs to pair (li - 1) / 2 (V_f and K_{f+1}); K_0 has a
    barrier of its own.  Of li copies, all that were begun have to be in the pairs waited for,
    and the others complete: a V that no K follows is completed by hand at the end."""
    part = body(source("kv_chunk.cu"), "else if (warp == 0) {")
    first, last = re.search(r"for \(int i = max\(0, ([^;]*) - PAIRS\); i < ([^;]*); \+\+i\) mbar_land\(&sh.pair", part).groups()
    assert first == last
    for li in range(1, 30):
        begun = {(i - 1) // 2 for i in range(1, li)}
        waited = set(range(eval(last.replace("/", "//"), {"li": li})))
        by_hand = (li - 1) // 2
        whole = {f for f in begun if {2 * f + 1, 2 * f + 2} <= set(range(li)) or f == by_hand}
        assert begun <= waited and waited <= whole, li
