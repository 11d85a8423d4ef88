"""Forking, growing, freeing, compacting and copying pages against oracle/cache.py: tables, lengths, counts and the
pool's bytes are equal."""
import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from cache_cases import ids, same_pool, to_gpu
from oracle import cache as oc

pytestmark = pytest.mark.gpu


def refs_of(table, lengths, ps, pages, held=()):
    """What the rows hold, and pages that something else holds besides."""
    refs = np.zeros(pages, np.int32)
    for row, L in zip(table, lengths):
        for p in row[:(max(0, min(L, table.shape[1] * ps)) + ps - 1) // ps]:
            if 0 <= p < pages:
                refs[p] += 1
    for p in held:
        refs[p] += 1
    return refs


def fork(pool, table, lengths, refs, parent=None, keep=None, grow=None, in_place=False):
    cache = to_gpu(pool)
    S = len(lengths) if parent is None else len(parent)
    status = torch.zeros(S, dtype=torch.int32, device="cuda:0")
    opt = {n: None if x is None else ids(x) for n, x in (("parent", parent), ("keep", keep), ("grow", grow))}
    got = mdss.cache_fork(cache, ids(table), ids(lengths), ids(refs), row_status=status, **opt)
    want = oc.fork(pool, table, lengths, refs, parent, keep, grow)
    torch.cuda.synchronize()
    for g, w, name in zip(got, want, ("table", "lengths", "refs")):
        np.testing.assert_array_equal(g.cpu().numpy(), w, err_msg=name)
    assert {i for i in range(S) if status[i].item() == 64} == want[3]
    assert sum(1 for x in status.tolist() if x) == len(want[3])
    same_pool(cache, pool)
    return want[:3]


def start(S, ps, pages, width, longest, rng, layers=2, heads=2, d=64):
    lengths = [int(x) for x in rng.integers(0, longest + 1, S)]
    order, at = rng.permutation(pages), 0
    table = np.full((S, width), -1, np.int32)
    for s, L in enumerate(lengths):
        n = (L + ps - 1) // ps
        table[s, :n] = order[at:at + n]
        at += n
    return oc.new_pool(layers, pages, heads, d, ps, rng), table, lengths


@pytest.mark.parametrize("seed", range(8))
def test_steps_of_a_search(seed):
    """Random parents, truncation and growth, step after step on the same pool."""
    rng = np.random.default_rng([20, seed])
    ps = [16, 32, 64, 16][seed % 4]
    S = [1, 5, 12, 40][seed % 4]
    pages = S * 12 + 40
    pool, table, lengths = start(S, ps, pages, 12, 5 * ps, rng, d=[64, 96, 128, 256][seed % 4])
    refs = refs_of(table, lengths, ps, pages, held=rng.integers(0, pages, 3))
    for step in range(6):
        n = len(lengths)
        out = max(1, n + int(rng.integers(-2, 3))) if step else n
        parent = rng.integers(-1, n, out)
        keep = rng.integers(0, 6 * ps, out) if rng.random() < 0.5 else None
        grow = rng.choice([0, 1, 1, 3, ps, 2 * ps + 1], out) if rng.random() < 0.8 else None
        if grow is not None and keep is None:
            keep = np.minimum(np.array([max(0, lengths[p]) if p >= 0 else 0 for p in parent]), 6 * ps)
        table, lengths, refs = fork(pool, table, list(lengths), refs, parent, keep, grow)
        lengths = [int(x) for x in lengths]


def test_growth_only_and_no_change():
    rng = np.random.default_rng(21)
    ps, pages = 16, 60
    pool, table, lengths = start(6, ps, pages, 8, 60, rng)
    refs = refs_of(table, lengths, ps, pages)
    fork(pool, table, lengths, refs)
    fork(pool, table, lengths, refs, grow=[1] * 6)
    fork(pool, table, lengths, refs, grow=[0, 16, 17, 1, 0, 40])
    fork(pool, table, lengths, refs, keep=[0, 16, 17, 1, 1000, -3])
    fork(pool, table, lengths, refs, parent=[-1] * 6)
    fork(pool, table, lengths, refs, parent=[])


def test_beams_of_one_prompt():
    """A prompt becomes eight beams on one partly filled page: seven copies, the last beam keeps it."""
    rng = np.random.default_rng(22)
    ps, pages = 16, 20
    pool = oc.new_pool(3, pages, 1, 64, ps, rng)
    table = np.full((1, 6), -1, np.int32)
    table[0, :3] = [7, 3, 11]
    refs = refs_of(table, [40], ps, pages)
    t, n, r = fork(pool, table, [40], refs, parent=[0] * 8, grow=[1] * 8)
    assert r[11] == 1 and t[7, 2] == 11 and r[7] == 8 and sorted(t[:7, 2]) == [0, 1, 2, 4, 5, 6, 8]
    # the same with a row that does not grow: it holds the page too, so all eight copy
    fork(pool, table, [40], refs, parent=[0] * 9, grow=[1] * 8 + [0])
    # whole pages are shared and the growth takes new ones
    fork(pool, table, [32], refs_of(table, [32], ps, pages), parent=[0] * 4, grow=[2] * 4)


def test_too_few_pages_and_too_narrow_a_table():
    rng = np.random.default_rng(23)
    ps, pages = 16, 9
    pool = oc.new_pool(1, pages, 1, 64, ps, rng)
    table = np.array([[0, 1, -1], [2, 3, 4], [5, -1, -1]], np.int32)
    lengths = [20, 48, 16]
    refs = refs_of(table, lengths, ps, pages)
    fork(pool, table, lengths, refs, parent=[0, 0, 1, 2], grow=[1, 13, 0, 17])   # one page too many
    fork(pool, table, lengths, refs, parent=[0, 0, 1, 2], grow=[1, 1, 1, 17])    # row 2 passes the table
    fork(pool, table, lengths, refs, parent=[0, 0, 1, 2], grow=[1, 0, 0, 16])
    # what this call frees is not yet handed out
    full = np.ones(pages, np.int32)
    fork(pool, table, lengths, full, parent=[-1, 1, 2], grow=[0, 0, 1])


def test_ids_out_of_range_and_odd_rows():
    rng = np.random.default_rng(24)
    ps, pages = 16, 10
    pool = oc.new_pool(1, pages, 2, 64, ps, rng)
    table = np.array([[0, 99, 2], [-5, 4, -1]], np.int32)
    lengths = [40, 20]
    refs = refs_of(table, lengths, ps, pages)
    fork(pool, table, lengths, refs, parent=[0, 1, 0, 7, -9], grow=[1, 1, 1, 1, 1])
    fork(pool, table, [-4, 1000], refs_of(table, [-4, 1000], ps, pages), parent=[1, 0], keep=[20, 20], grow=[1, 1])


def test_many_rows_and_a_large_pool():
    rng = np.random.default_rng(25)
    ps, pages, S = 16, 70000, 1500
    pool, table, lengths = start(S, ps, pages, 5, 50, rng, layers=1, heads=1)
    refs = refs_of(table, lengths, ps, pages, held=rng.integers(0, pages, 1000))
    table, lengths, refs = fork(pool, table, lengths, refs, parent=rng.integers(-1, S, 1300), grow=rng.integers(0, 30, 1300))


@pytest.mark.parametrize("pages,share", [(1, 0.5), (7, 0.5), (64, 0.3), (1023, 0.5), (1024, 0.6), (1025, 0.1), (5000, 0.4),
                                         (300, 0.0), (300, 1.0)])
def test_compact(pages, share):
    rng = np.random.default_rng([26, pages])
    ps, S = 16, 4
    pool = oc.new_pool(2, pages, 1, 64, ps, rng)
    used = rng.permutation(pages)[:int(pages * share)]
    width = max(1, len(used) // S) + 1
    table, lengths = np.full((S, width), -1, np.int32), []
    for s in range(S):
        mine = used[s::S][:width]
        table[s, :len(mine)] = mine
        lengths.append(max(0, len(mine) * ps - int(rng.integers(0, ps))))
    table[0, -1] = 5  # past the row's tokens
    lengths[0] = min(lengths[0], (width - 1) * ps)
    refs = refs_of(table, lengths, ps, pages)
    refs[used] = np.maximum(refs[used], rng.integers(1, 4, len(used)))
    cache = to_gpu(pool)
    got = mdss.cache_compact(cache, ids(table), ids(lengths), ids(refs))
    want = oc.compact(pool, table, lengths, refs)
    torch.cuda.synchronize()
    for g, w in zip(got[:2], want[:2]):
        np.testing.assert_array_equal(g.cpu().numpy(), w)
    assert int(got[2]) == want[2]
    same_pool(cache, pool)


@pytest.mark.parametrize("heads,d,ps", [(1, 64, 16), (3, 96, 32), (5, 256, 64)])
def test_copy(heads, d, ps):
    rng = np.random.default_rng(27)
    pool = oc.new_pool(3, 12, heads, d, ps, rng)
    cache = to_gpu(pool)
    mdss.cache_copy(cache, ids([3, 0, 99, 4, 3]), ids([7, 8, 2, -1, 9]))
    for n in pool:
        for a, b in ((3, 7), (0, 8), (3, 9)):
            pool[n][:, b] = pool[n][:, a]
    same_pool(cache, pool)
    mdss.cache_copy(cache, ids([]), ids([]))
    same_pool(cache, pool)


def test_fork_in_a_graph():
    rng = np.random.default_rng(28)
    ps, pages = 16, 80
    pool, table, lengths = start(6, ps, pages, 6, 60, rng)
    refs = refs_of(table, lengths, ps, pages)
    cache = to_gpu(pool)
    args = (ids(table), ids(lengths), ids(refs))
    parent, grow = ids([0, 0, 1, 3, 3, 5]), ids([1] * 6)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = mdss.cache_fork(cache, *args, parent=parent, grow=grow)
    want = oc.fork(pool, table, lengths, refs, [0, 0, 1, 3, 3, 5], None, [1] * 6)
    for _ in range(3):
        for x in got:
            x.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            np.testing.assert_array_equal(g.cpu().numpy(), w)
        torch.randn(1000, device="cuda:0").sum().item()
    same_pool(cache, pool)
