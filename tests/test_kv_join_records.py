"""The joining kernel of attention over the paged cache takes its addresses from records that
the CTAs of the kernel before it leave.  A CTA whose wait gives up stops there, so that its
record has to stand before the first wait; and where the kernel before was not launched,
there are none.  Neither can be brought about on a healthy GPU: the sources are read.  No GPU."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_02474_gb300", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


@pytest.mark.parametrize("name,role", [("kv_decode.cu", "if (warp == C::WARPS) {"), ("kv_chunk.cu", "if (warp == 3) {")])
def test_the_record_stands_before_the_first_wait(name, role):
    text = source(name)
    assert text.count(role) == 1
    part = text[text.index(role):]                 # the warp that walks the pieces
    record = part.index("kv_leave_join(")
    assert record < re.search(r"\b(mbar_wait|wait_all)\(", part).start()
    assert re.search(r"\b(for|while)\s*\(", part).start() > record
    assert "kv_leave_join(" not in text[:text.index(role)]


@pytest.mark.parametrize("name", ["kv_decode.cu", "kv_chunk.cu"])
def test_no_join_without_the_kernel_before_it(name):
    text = source(name)
    calls = re.findall(r"([^;{}]*)\blaunch_kv_join\(", text)
    assert len(calls) == 1 and "if (launched == cudaSuccess)" in calls[0]
    assert len(re.findall(r"launched = echo::launch_chained\(", text)) == 1
