"""What rows of the cache share, against oracle/cache.py."""
import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from cache_cases import ids
from oracle import cache as oc
from shared_cases import Groups

pytestmark = pytest.mark.gpu


def pool_of(pages, ps):
    return mdss.PagedCache.empty(1, pages, 1, 64, ps)


def check(cache, starts, table, lengths, groups, least=0, uniform=False):
    T = int(starts[-1])
    tokens, rows = mdss.cache_shared(cache, T, None if uniform else ids(starts), ids(table), ids(lengths), ids(groups), least=least)
    want, want_rows = oc.shared(cache.pages, cache.page_size, starts, table, lengths, groups, least)
    np.testing.assert_array_equal(tokens.cpu().numpy(), want)
    np.testing.assert_array_equal(rows.cpu().numpy(), want_rows)
    return want, want_rows


@pytest.mark.parametrize("ps", [16, 64, 128, 256])
@pytest.mark.parametrize("seed", range(3))
def test_random_groups(ps, seed):
    rng = np.random.default_rng([ps, seed])
    rows = []
    for _ in range(12):
        prefix = int(rng.choice([0, 1, 63, 64, 65, 128, 300, 1000, 2049]))
        W = int(rng.choice([1, 1, 2, 3, 5, 8]))
        members = [(int(n), None if rng.random() < 0.15 else int(n + rng.choice([0, 0, 1, 5, 100, 300]))) for n in rng.integers(0, 6, W)]
        rows.append((prefix, members))
    c = Groups(rows, ps, rng)
    for s in rng.integers(0, len(c.new), 6):  # rows that went their own way earlier, and ids outside the pool
        j = int(rng.integers(0, c.table.shape[1]))
        c.table[s, j:] = np.where(c.table[s, j:] >= 0, rng.choice([c.pages - 1, c.pages - 2, c.pages + 5, -7]), -1)
    cache = pool_of(c.pages, ps)
    for least in (0, 1, 64, 200, 5000):
        check(cache, c.starts, c.table, c.lengths, c.groups, least)
    # rows before the first group and after the last one are in none
    inner = c.groups[1:-1]
    check(cache, c.starts, c.table, c.lengths, inner)
    check(cache, c.starts, c.table, c.lengths, [0])
    check(cache, c.starts, c.table, c.lengths, [3, 3, 3, 3])


def test_uniform_new_tokens():
    rng = np.random.default_rng(2)
    c = Groups([(500, [(2, 30), (2, 70), (2, 2)]), (64, [(2, 2), (2, 2)]), (200, [(2, 9)])], 16, rng)
    want, _ = check(pool_of(c.pages, 16), c.starts, c.table, c.lengths, c.groups, uniform=True)
    assert want.tolist() == [448] * 3 + [64] * 2 + [0]


def test_borders():
    """Shared tokens end with the pages, with a row's tokens, or before its new ones."""
    rng = np.random.default_rng(3)
    ps = 16
    c = Groups([(640, [(1, 100), (1, 1)]), (640, [(5, 4), (1, 200)]), (64, [(1, 0), (1, 1)]), (127, [(1, 30)] * 3)], ps, rng)
    want, rows = check(pool_of(c.pages, ps), c.starts, c.table, c.lengths, c.groups)
    assert want.tolist() == [640] * 2 + [576] * 2 + [0] * 2 + [64] * 3


def test_many_rows_and_pages():
    """A group of more rows than a workgroup's threads, tables longer than one step, the difference anywhere."""
    rng = np.random.default_rng(4)
    S, width, ps = 2100, 700, 16
    table = np.tile(rng.permutation(width).astype(np.int32), (S, 1))
    lengths = np.full(S, width * ps, np.int32)
    starts = np.arange(S + 1, dtype=np.int32)
    cache = pool_of(width + 1, ps)
    for row, at in ((2099, 699), (1030, 513), (5, 256), (64, 255), (0, 63), (700, 0)):
        table[row, at] = width
        check(cache, starts, table, lengths, [0, S])
        check(cache, starts, table, lengths, [0, 1, 1500, S])
    lengths[rng.integers(0, S, 40)] = rng.integers(-5, 3000, 40)
    check(cache, starts, table, lengths, [0, S])
    check(cache, starts, table, lengths, list(range(0, S + 1, 3)), 700)


def test_groups_that_are_none():
    """Bounds that do not ascend within the rows: nothing is read through them."""
    c = Groups([(200, [(1, 5)] * 4)], 16, np.random.default_rng(5))
    cache = pool_of(c.pages, 16)
    for groups in ([-3, 4], [0, 9], [3, 1], [5, 5], [1 << 30, (1 << 31) - 1]):
        tokens, rows = mdss.cache_shared(cache, c.T, ids(c.starts), ids(c.table), ids(c.lengths), ids(groups))
        torch.cuda.synchronize()
        if not 0 <= groups[0] <= groups[1] <= 4:
            assert rows.tolist() == [[0, 0, -1, 0]]
    tokens, rows = mdss.cache_shared(cache, c.T, ids(c.starts), ids(c.table), ids(c.lengths), ids([0, 9, 4]))
    assert tokens.tolist() == [0] * 4 and rows.tolist() == [[0, 0, -1, 0]] * 2
    tokens, rows = mdss.cache_shared(cache, 0, ids([0]), ids(np.zeros((0, 3))), ids([]), ids([0, 0]))
    assert tokens.numel() == 0 and rows.tolist() == [[0, 0, -1, 0]]


def test_a_captured_graph():
    c = Groups([(640, [(1, 100), (1, 50), (1, 300)]), (300, [(1, 5)] * 4)], 16, np.random.default_rng(6))
    cache, starts, table, lengths, groups = pool_of(c.pages, 16), ids(c.starts), ids(c.table), ids(c.lengths), ids(c.groups)
    mdss.cache_shared(cache, c.T, starts, table, lengths, groups)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = mdss.cache_shared(cache, c.T, starts, table, lengths, groups)
    for row, at in ((0, 30), (5, 7), (1, 4)):
        table[row, at] = c.pages - 1
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = mdss.cache_shared(cache, c.T, starts, table, lengths, groups)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
