"""Host bookkeeping of shared pages (pipeline.PageTable).  No GPU."""
import pytest

from paper_2608_02474_gb300.pipeline import PageTable


def test_pages_are_taken_grown_and_given_back():
    t = PageTable(6, 16)
    t.open(7)
    t.open(9)
    t.extend({7: 16, 9: 1})
    t.extend({7: 1, 9: 15})                            # a page more for 7, none for 9
    assert t.pages == {7: [0, 2], 9: [1]} and t.lens == {7: 17, 9: 16}
    with pytest.raises(MemoryError):
        t.extend({7: 32, 9: 32})                       # four pages, three free: nothing changes
    assert t.pages == {7: [0, 2], 9: [1]} and t.lens == {7: 17, 9: 16} and len(t.free) == 3
    t.close(7)
    assert sorted(t.free) == [0, 2, 3, 4, 5] and 7 not in t.lens
    t.open(7)
    t.extend({7: 5 * 16})
    assert sorted(t.pages[7]) == [0, 2, 3, 4, 5] and not t.free


def test_opening_twice_and_growing_a_closed_clip():
    t = PageTable(2, 16)
    t.open(1)
    with pytest.raises(ValueError):
        t.open(1)
    t.close(1)
    with pytest.raises(KeyError):
        t.extend({1: 1})
    t.extend({})
    assert t.lens == {}
