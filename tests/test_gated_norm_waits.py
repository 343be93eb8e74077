"""The gated norm's waits for its rows where one of them gives up.  The lanes of a warp may then
see different things (the copy's barrier complete, the time limit, another warp's flag), and a
warp-wide exchange that some of its lanes do not come to never ends.  A wait that gives up cannot be
brought about on a healthy GPU: the source is read.  No GPU."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_02474_gb300", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_a_warp_gives_up_as_one():
    """What a wait found is the warp's and not a lane's."""
    text = source("gated_norm.cu")
    waits = re.findall(r"([^;{}]*)\bmbar_wait\(", text)
    assert waits and all(re.search(r"__all_sync\(0xffffffffu, [^()]*$", w) for w in waits), waits


def test_exchanges_are_no_operands_of_a_choice():
    """No lane's own value decides whether it comes to a warp-wide exchange."""
    text = source("gated_norm.cu")
    assert text.count("__shfl") > 5 and not re.findall(r"(?:\?|:|&&|\|\|)\s*__(?:shfl|all|any|ballot)[^;]*;", text)
