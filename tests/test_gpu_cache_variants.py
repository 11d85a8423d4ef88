"""Every compiled form of the attention kernels against oracle/cache.py: head sizes, types, row tiles, whole and in splits, NaN
codes in calls that are split.  Bound: tests/test_gpu_cache_attention.py's."""
import numpy as np
import pytest

import paper_2410_18234_amd as mdss
from cache_cases import ids, tables, to_gpu
from oracle import cache as oc
from test_gpu_cache_attention import fill, queries, run

pytestmark = pytest.mark.gpu

ROWS = [(1, 4), (3, 8), (7, 8), (10, 16)]  # new tokens and group: one, two, four row tiles (many rows where d = 256), many rows


def splits_taken(pool, T, S, width, heads_q, uniform, new=0, longest=0):
    c = to_gpu({n: x[:, :1] for n, x in pool.items()})
    return mdss.load_library().mdss_workspace_bytes_attention(c._ref, T, S, width, heads_q, uniform, new, longest) > 0


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("n,group", [(33, 1), (70, 2), (40, 8)])
def test_many_rows(d, n, group, kind):
    rng = np.random.default_rng([d, n, group])
    ps, new, lengths = 16, [n, n - 1, n], [n, n + 150, n + 3]
    pages = sum((x + ps - 1) // ps for x in lengths)
    pool = oc.new_pool(1, pages, 2, d, ps)
    fill(pool, rng)
    q, q64 = queries(rng, (sum(new), 2 * group, d), kind)
    table = tables(lengths, ps, pages, rng)
    run(pool, q, q64, new, lengths, table, kind)
    run(pool, q, q64, new, lengths, table, kind, max_new=1000, max_length=max(lengths))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("n,group", ROWS)
def test_splits(d, n, group, kind):
    rng = np.random.default_rng([d, n, group, 1])
    ps, new, lengths = 32, [n, 1, n], [5000, 37, 2600]
    pages = sum((x + ps - 1) // ps for x in lengths)
    pool = oc.new_pool(1, pages, 1, d, ps)
    fill(pool, rng)
    q, q64 = queries(rng, (sum(new), group, d), kind)
    table = tables(lengths, ps, pages, rng)
    assert splits_taken(pool, sum(new), 3, table.shape[1], group, 0, n)
    run(pool, q, q64, new, lengths, table, kind, max_new=n)
    run(pool, q, q64, new, lengths, table, kind, max_new=n, max_length=3000)  # the last split takes what lies past the hint
    run(pool, q[:n], q64[:n], [n], lengths[:1], table[:1], kind, uniform=True)


@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("n,group", ROWS)
def test_nan_codes_in_splits(d, n, group):
    rng = np.random.default_rng([d, n, group, 2])
    ps, lengths = 32, [4500, 3000]
    pages = sum((x + ps - 1) // ps for x in lengths)
    pool = oc.new_pool(1, pages, 1, d, ps)
    fill(pool, rng)
    table = tables(lengths, ps, pages, rng)

    def spoil(name, s, token, element):
        codes = oc.tokens_of(pool, name, 0, table[s, token // ps], 0).copy()
        codes[token % ps, element] = 0x7f
        oc.put_tokens(pool, name, 0, table[s, token // ps], 0, codes)

    spoil("v", 0, 4499, 3)        # the last row's own token
    spoil("v", 0, 1000, d - 1)    # seen by all, in one element
    spoil("k", 1, 2999, d // 2)   # the last row's own token, in all elements
    q, q64 = queries(rng, (2 * n, group, d), "bf16")
    assert splits_taken(pool, 2 * n, 2, table.shape[1], group, 1)
    run(pool, q, q64, [n, n], lengths, table, "bf16", uniform=True)


@pytest.mark.parametrize("n,group", ROWS)
@pytest.mark.parametrize("length", [300, 5000])
def test_calls_repeat_themselves(n, group, length):
    rng = np.random.default_rng([n, length])
    pool = oc.new_pool(1, 320, 2, 128, 32)
    fill(pool, rng)
    q, _ = queries(rng, (2 * n, 2 * group, 128), "bf16")
    cache = to_gpu(pool)
    table = ids(tables([length, length // 2], 32, 320, rng))
    args = (q, cache, 0, None, table, ids([length, length // 2]))
    first = mdss.cache_attention(*args).clone()
    for _ in range(5):
        assert (mdss.cache_attention(*args) == first).all()


@pytest.mark.parametrize("scale", [0.25, 0.5, 1.0, 4.0, 16.0])
@pytest.mark.parametrize("n,group", ROWS)
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_scores_of_wide_spread(d, n, group, scale):
    """Normal keys and queries, scores from 2 to 16 times as far apart as usual and more: from many tokens that count to one."""
    rng = np.random.default_rng([d, n, int(4 * scale)])
    lengths = [700, 650]
    pool = oc.new_pool(1, 45, 1, d, 32)
    fill(pool, rng)
    q, q64 = queries(rng, (2 * n, group, d), "f16")
    run(pool, q, q64, [n, n], lengths, tables(lengths, 32, 45, rng), "f16", uniform=True, scale=scale)
