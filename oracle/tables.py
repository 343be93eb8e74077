"""Page tables and slot maps of a step, page by page as a person would keep them.

TEST INFRASTRUCTURE ONLY (see the package header).

An addition of this build, not of the paper: slots of sequences share a stack of free
pages.  extend() gives each named slot, in order, the pages that its new rows need, from the
top of the stack; shorten() takes tokens back, and the pages that nothing needs any more,
so that shortening by the same rows undoes extending.  All or nothing.

Pins: a hand-worked run; extend then shorten restores the stack, entry by entry; pages are
free or in one table, never both; a refused call changes nothing.
"""
from __future__ import annotations

LIMIT = 2 ** 31 - 128


class Tables:
    def __init__(self, n_pages, page, n_slots, max_pages, free=None):
        self.page, self.max_pages = page, max_pages
        self.free = list(range(n_pages - 1, -1, -1)) if free is None else list(free)
        self.pages = [[] for _ in range(n_slots)]
        self.lens = [0] * n_slots

    def _named(self, slots):
        return len(set(slots)) == len(slots) and all(0 <= s < len(self.lens) for s in slots)

    def extend(self, slots, rows, n_rows):
        """(lens, row0, [(place, pos, seq)] of n_rows rows), or None where it cannot be served."""
        if not self._named(slots) or min(rows, default=0) < 0 or sum(rows) > n_rows:
            return None
        most = min(self.max_pages * self.page, LIMIT)
        if any(self.lens[s] + n > most for s, n in zip(slots, rows)):
            return None
        need = [-(-(self.lens[s] + n) // self.page) - len(self.pages[s]) for s, n in zip(slots, rows)]
        if sum(need) > len(self.free):
            return None
        lens, row0, maps = [], [0], []
        for b, (s, n, k) in enumerate(zip(slots, rows, need)):
            for _ in range(k):
                self.pages[s].append(self.free.pop())
            for p in range(self.lens[s], self.lens[s] + n):
                maps.append((self.pages[s][p // self.page] * self.page + p % self.page, p, b))
            self.lens[s] += n
            lens.append(self.lens[s])
            row0.append(row0[-1] + n)
        return lens, row0, maps + [(-1, -1, -1)] * (n_rows - len(maps))

    def shorten(self, slots, rows):
        if not self._named(slots) or min(rows, default=0) < 0:
            return False
        given = []
        for s, n in zip(slots, rows):
            self.lens[s] -= min(n, self.lens[s])
            keep = -(-self.lens[s] // self.page)
            given += self.pages[s][keep:]
            del self.pages[s][keep:]
        self.free += reversed(given)
        return True
