"""Shared by the tests of prefixes: tables whose rows share their leading pages, group by group."""
import numpy as np

from cache_cases import starts_of


def up(a, b):
    return -(-a // b)


class Groups:
    """rows: for each group (prefix, [(new tokens, tokens past the prefix), ...]); a row of None tokens holds nothing.  What the
    prefix holds of whole pages is common to the group's rows, what comes after is each row's own."""

    def __init__(self, rows, ps, rng, extra=1, spare=2):
        self.ps, self.new, self.lengths, self.groups = ps, [], [], [0]
        lists, count = [], 0
        for prefix, members in rows:
            common = prefix // ps
            mine = list(range(count, count + common))
            count += common
            for n, more in members:
                L = 0 if more is None else prefix + more
                own = max(0, up(L, ps) - common)
                lists.append(([] if more is None else mine) + list(range(count, count + own)))
                count += own
                self.new.append(n)
                self.lengths.append(L)
            self.groups.append(len(self.new))
        self.pages = count + spare
        order = rng.permutation(self.pages)
        self.table = np.full((len(lists), max(len(x) for x in lists) + extra), -1, np.int32)
        for s, x in enumerate(lists):
            self.table[s, :len(x)] = order[x]
        self.starts = starts_of(self.new)
        self.T = int(self.starts[-1])
