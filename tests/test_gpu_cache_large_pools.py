"""Compaction and forks beyond the sizes that one workgroup takes (8192 pages, 16384 table entries), against oracle/cache.py:
tables, lengths, counts and bytes are equal.  Pages are told apart by their bytes."""
import numpy as np
import pytest

import paper_2410_18234_amd as mdss
from cache_cases import ids, same_pool, to_gpu
from oracle import cache as oc
from test_gpu_cache_pages import fork, refs_of

pytestmark = pytest.mark.gpu

PS = 16


def marked_pool(pages, layers=1):
    pool = oc.new_pool(layers, pages, 1, 64, PS)
    at = np.arange(pages)
    for layer in range(layers):
        for n, step in (("k", 1), ("v", 7)):
            pool[n][layer, :, 0, 0, 0] = ((at * step + layer) % 251).astype(np.uint8)[:, None, None] if n == "k" else \
                ((at * step + layer) % 251).astype(np.uint8)[:, None]
            pool[n][layer, :, 0, 0, 1] = (at // 251 % 251).astype(np.uint8)[:, None, None] if n == "k" else \
                (at // 251 % 251).astype(np.uint8)[:, None]
            pool[n + "_exp"][layer, :, 0] = at % 81 - 40
    return pool


def rows_over(used, S, width, rng, spare=0):
    """The used pages dealt out to S rows: (table, lengths)."""
    table, lengths = np.full((S, width), -1, np.int32), []
    for s in range(S):
        mine = used[s::S][:width - spare]
        table[s, :len(mine)] = mine
        lengths.append(max(0, len(mine) * PS - int(rng.integers(0, PS))))
    return table, lengths


def compact(pool, table, lengths, refs):
    cache = to_gpu(pool)
    got = mdss.cache_compact(cache, ids(table), ids(lengths), ids(refs))
    want = oc.compact(pool, table, lengths, refs)
    for g, w in zip(got[:2], want[:2]):
        np.testing.assert_array_equal(g.cpu().numpy(), w)
    assert int(got[2]) == want[2]
    same_pool(cache, pool)


@pytest.mark.parametrize("pages", [8192, 8193, 9 * 1024, 70000])
@pytest.mark.parametrize("used", ["none", "all", "low", "high", "half", "chunks", "few"])
def test_compact(pages, used):
    rng = np.random.default_rng([pages, len(used)])
    order = rng.permutation(pages)
    held = {"none": order[:0], "all": order, "low": np.arange(3000), "high": np.arange(pages - 3000, pages), "half": order[:pages // 2],
            "chunks": order[:4096], "few": order[:3]}[used]
    S = 8
    table, lengths = rows_over(held, S, max(1, -(-len(held) // S)), rng)
    refs = refs_of(table, lengths, PS, pages)
    refs[held] = np.maximum(refs[held], rng.integers(1, 4, len(held)))
    compact(marked_pool(pages), table, lengths, refs)


@pytest.mark.parametrize("S,width", [(1, 16385), (300, 60), (4096, 5)])
def test_compact_of_few_pages_and_many_entries(S, width):
    """A small pool whose pages many rows share."""
    rng = np.random.default_rng([S, width])
    pages = 500
    order = rng.permutation(pages)[:200]
    table = order[rng.integers(0, 200, (S, width))].astype(np.int32)
    lengths = [int(x) for x in rng.integers(0, width * PS + 1, S)]
    compact(marked_pool(pages, layers=3), table, lengths, refs_of(table, lengths, PS, pages))


def test_tables_of_several_batches_follow_together():
    """Rows do not change what is moved, so a table that holds pages besides is stacked on; a row of all ids comes back as the map."""
    rng = np.random.default_rng(5)
    pages, S = 9000, 4
    order = rng.permutation(pages)
    table, lengths = rows_over(order[:2000], S, 500, rng)
    other, other_lengths = rows_over(order[2000:2600], S, 500, rng)
    all_ids = np.arange(pages, dtype=np.int32).reshape(-1, 500)
    refs = refs_of(np.concatenate((table, other)), lengths + other_lengths, PS, pages)
    pool = marked_pool(pages)
    cache = to_gpu(pool)
    stacked = np.concatenate((table, other, all_ids))
    got, now, used = mdss.cache_compact(cache, ids(stacked), ids(lengths + other_lengths + [500 * PS] * len(all_ids)), ids(refs))
    got, held = got.cpu().numpy(), refs > 0
    to = got[2 * S:].reshape(-1)
    assert int(used) == held.sum() and np.array_equal(np.sort(to[held]), np.arange(int(used))) and (to[~held] == -1).all()
    for before, after, n in ((table, got[:S], lengths), (other, got[S:2 * S], other_lengths)):
        for s in range(S):
            k = (n[s] + PS - 1) // PS
            np.testing.assert_array_equal(after[s, :k], to[before[s, :k]])
    now_k = cache.k.cpu().numpy()
    np.testing.assert_array_equal(now_k[:, to[held]], pool["k"][:, held])


@pytest.mark.parametrize("pages,S,width", [(9000, 40, 12), (500, 1200, 3), (300, 200, 90)])
@pytest.mark.parametrize("case", ["parents", "own", "mixed", "none", "no growth", "keep"])
def test_fork(pages, S, width, case):
    rng = np.random.default_rng([pages, S, len(case)])
    room = pages // 2
    lengths = [int(x) for x in rng.integers(0, min(width * PS - 20, max(17, room // S * PS)) + 1, S)]
    table, at, order = np.full((S, width), -1, np.int32), 0, rng.permutation(pages)
    for s, L in enumerate(lengths):
        n = (L + PS - 1) // PS
        if at + n > room:  # the rest share
            lengths[s], table[s] = lengths[0], table[0]
            continue
        table[s, :n] = order[at:at + n]
        at += n
    refs = refs_of(table, lengths, PS, pages, held=order[room:room + 20])
    pool = marked_pool(pages)
    grow = rng.choice([0, 0, 0, 1, 3], S)
    own = np.arange(S)
    some = np.where(rng.random(S) < 0.5, own, rng.integers(-1, S, S))
    if case == "parents":
        fork(pool, table, lengths, refs, parent=rng.integers(-1, S, S - 3), grow=grow[:S - 3])
    elif case == "own":
        fork(pool, table, lengths, refs, parent=own, grow=grow)
    elif case == "mixed":
        fork(pool, table, lengths, refs, parent=some, grow=grow)
    elif case == "none":
        fork(pool, table, lengths, refs, grow=grow)
    elif case == "no growth":
        fork(pool, table, lengths, refs, parent=some)
    else:  # a draft is kept, what was rejected is cut, the rest is given back
        keep = np.maximum(np.array(lengths) - rng.integers(0, 40, S), 0)
        fork(pool, table, lengths, refs, parent=np.where(own % 4 == 1, own, -1), keep=keep, grow=grow)
        fork(pool, table, lengths, refs, keep=keep, grow=grow)


def test_fork_of_a_pool_beyond_the_near_counts():
    """More than 2^18 pages: the free pages' counts stay in memory."""
    rng = np.random.default_rng(9)
    pages, S, width = (1 << 18) + 3000, 50, 40
    refs = np.ones(pages, np.int32)  # most pages are held by something else
    free = np.concatenate((rng.choice(pages - 5, 400, replace=False), np.arange(pages - 5, pages)))
    refs[free] = 0
    held = rng.choice(np.setdiff1d(np.arange(pages), free), 600, replace=False)
    lengths = [int(x) for x in rng.integers(1, 12 * PS, S)]
    table, at = np.full((S, width), -1, np.int32), 0
    for s, L in enumerate(lengths):
        n = (L + PS - 1) // PS
        table[s, :n] = held[at:at + n]
        at += n
    table_, lengths_, refs_ = fork(marked_pool(pages), table, lengths, refs, parent=rng.integers(-1, S, S), grow=rng.integers(0, 60, S))
    assert refs_.sum() > 0 and (lengths_ > 0).any()
