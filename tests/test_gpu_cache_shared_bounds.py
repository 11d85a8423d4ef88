"""Groups whose bounds do not ascend (lists padded with zeros, bounds out of the rows, groups that overlap) leave the others as they are: what
rows share, and attention over it."""
import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from cache_cases import ids, to_gpu
from oracle import cache as oc
from shared_cases import Groups
from test_gpu_cache_attention import check, fill, queries
from test_gpu_cache_shared import check as check_shared
from test_gpu_cache_shared import pool_of

pytestmark = pytest.mark.gpu

LISTS = [[0, 4, 8, 0, 0, 0], [0, 4, 8, 12, 0], [4, 8, 0, 0, 12], [0, 4, 2, 8, 12], [0, 8, 4, 12], [0, 0, 0, 4, 0, 8, 0, 12, 0], [-1, 4, 8, 13, 12, 12],
         [0, 4, 1 << 30, 8, 12], [12, 4, 8, 12], [8, 12, 0, 4], [0, 4, -(1 << 31), (1 << 31) - 1, 4, 8]]


@pytest.mark.parametrize("uniform", [False, True])
@pytest.mark.parametrize("groups", LISTS)
def test_what_rows_share(groups, uniform):
    rng = np.random.default_rng(1)
    c = Groups([(640, [(2, 2 + int(x)) for x in rng.integers(0, 200, 4)]) for _ in range(3)], 16, rng)
    check_shared(pool_of(c.pages, 16), c.starts, c.table, c.lengths, groups, uniform=uniform)


@pytest.mark.parametrize("G", [100, 2048, 2049, 5000, 65535])
def test_many_groups(G):
    """More groups than workgroups, with bounds out of order among them and at the end."""
    rng = np.random.default_rng(G)
    c = Groups([(130, [(1, 1 + int(x)) for x in rng.integers(0, 40, rng.integers(1, 6))]) for _ in range(300)], 16, rng)
    S = len(c.new)
    groups = np.sort(rng.integers(0, S + 1, G + 1)) if G < 3000 else np.concatenate((np.sort(rng.integers(0, S + 1, 2000)), np.zeros(G - 1999, int)))
    cache = pool_of(c.pages, 16)
    check_shared(cache, c.starts, c.table, c.lengths, groups.tolist())
    for i in rng.integers(0, G + 1, 9):
        groups[i] = rng.choice([-1, 0, S + 1, int(rng.integers(0, S + 1))])
    check_shared(cache, c.starts, c.table, c.lengths, groups.tolist())


@pytest.mark.parametrize("group", [4, 1])
@pytest.mark.parametrize("groups", LISTS)
def test_attention(groups, group):
    """Groups of several row tiles; the workspace holds no part of a row that the call did not write."""
    rng = np.random.default_rng([2, group])
    c = Groups([(640, [(10, 10 + int(x)) for x in rng.integers(0, 90, 4)]) for _ in range(3)], 16, rng)
    pool = oc.new_pool(1, c.pages, 1, 64, 16)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, group, 64), "f16")
    cache, starts, table, lengths = to_gpu(pool), ids(c.starts), ids(c.table), ids(c.lengths)
    shared = mdss.cache_shared(cache, c.T, starts, table, lengths, ids(groups))
    space = torch.full((1 << 20,), float("nan"), dtype=torch.float32, device="cuda:0").view(torch.uint8)
    out, lse = mdss.cache_attention_shared(q, cache, 0, starts, table, lengths, shared, want_lse=True, workspace=space)
    torch.cuda.synchronize()
    check(out, lse, oc.attention(pool, 0, q64, c.starts, c.table, c.lengths, 0.125), "f16", 64, 800)
