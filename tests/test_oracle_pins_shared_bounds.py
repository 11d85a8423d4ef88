"""Pins of what rows share by bounds that do not ascend, and why it is so: the row tiles of the groups are found by a search over their
first tokens, which have to ascend."""
import random

import numpy as np

from oracle import cache as oc


def test_bounds_by_hand():
    table = np.array([[5, 6, 7, 8, i] for i in range(6)], np.int32)
    lengths, starts = [70] * 6, 2 * np.arange(7)
    by = lambda groups: tuple(x.tolist() for x in oc.shared(10, 16, starts, table, lengths, groups))  # noqa: E731
    assert by([0, 2, 5, 0, 0]) == ([64] * 5 + [0], [[0, 4, 0, 64], [4, 6, 2, 64], [10, 0, -1, 0], [10, 0, -1, 0]])
    assert by([0, 3, 2, 6, 6]) == ([64] * 3 + [0] * 3, [[0, 6, 0, 64], [6, 0, -1, 0], [6, 0, -1, 0], [12, 0, -1, 0]])
    assert by([4, 9, 1, 3]) == ([0, 64, 64, 0, 0, 0], [[0, 0, -1, 0], [0, 0, -1, 0], [2, 4, 1, 64]])


def found(first, slot, group, tile):
    """The set of a slot past the sets' first ones, by 64 candidates a step."""
    lo, n = 0, len(first)
    while n > 1:
        step = (n + 63) >> 6
        hits = sum(lo + i * step < lo + n and first[lo + i * step] * group // tile <= slot for i in range(64))
        at = max(hits - 1, 0)
        lo, n = lo + at * step, min(step, n - at * step)
    return lo


def test_every_tile_of_a_group_has_a_slot():
    rng = random.Random(3)
    S = 40
    table = np.zeros((S, 8), np.int32)
    for _ in range(300):
        starts = np.cumsum([0] + [rng.randrange(0, 30) for _ in range(S)])
        groups = sorted(rng.randrange(0, S + 1) for _ in range(rng.choice([2, 5, 90])))
        for _ in range(rng.randrange(0, 4)):
            groups[rng.randrange(len(groups))] = rng.choice([0, -1, S + 1, rng.randrange(0, S + 1)])
        groups += [0] * rng.randrange(0, 3)
        rows = oc.shared(1, 16, starts, table, [128] * S, groups)[1]
        assert (np.diff(rows[:, 0]) >= 0).all()
        for group, tile in ((4, 128), (1, 16), (7, 64)):
            G, T = len(rows), int(starts[-1])
            there = {(g, 0) for g in range(G)}
            for slot in range(T * group // tile):
                g = found(rows[:, 0], slot, group, tile)
                there.add((g, 1 + slot - int(rows[g, 0]) * group // tile))
            for g in range(G):
                assert all((g, t) in there for t in range(-(-int(rows[g, 1]) * group // tile)))
