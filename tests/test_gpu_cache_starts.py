"""New tokens that begin past token 0 of the inputs (starts[0] > 0): the tokens before and after belong to no sequence."""
import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from cache_cases import ids, same_pool, starts_of, tables, to_gpu, to_pool
from oracle import cache as oc

pytestmark = pytest.mark.gpu

OFFSET, AFTER = 100, 5


def case(d, ps, seed):
    rng = np.random.default_rng([77, seed])
    new, lengths = [1, 20, 0, 3], [40, 150, 9, 3]
    pages = sum((x + ps - 1) // ps for x in lengths) + 2
    pool = oc.new_pool(1, pages, 2, d, ps)
    for n in ("k", "v"):
        pool[n][...] = oc.encode(rng.standard_normal(pool[n].shape) * 50.0)
        pool[n + "_exp"][...] = rng.integers(-8, -3, pool[n + "_exp"].shape)
    return pool, new, lengths, starts_of(new), tables(lengths, ps, pages, rng), rng


@pytest.mark.parametrize("group", [1, 4])
def test_attention(group):
    pool, new, lengths, starts, table, rng = case(64, 16, group)
    T = OFFSET + int(starts[-1]) + AFTER
    q = torch.from_numpy(rng.standard_normal((T, 2 * group, 64))).to(torch.bfloat16).cuda()
    cache = to_gpu(pool)
    mine = slice(OFFSET, T - AFTER)
    want = mdss.cache_attention(q[mine], cache, 0, ids(starts), ids(table), ids(lengths), max_new=20, max_length=150)
    out = torch.full_like(q, 3.0)
    mdss.cache_attention(q, cache, 0, ids(starts + OFFSET), ids(table), ids(lengths), max_new=20, max_length=150, out=out)
    assert torch.equal(out[mine], want)
    assert bool((out[:OFFSET] == 3.0).all()) and bool((out[T - AFTER:] == 3.0).all())


@pytest.mark.parametrize("ps", [16, 64])
def test_append(ps):
    pool, new, lengths, starts, table, rng = case(128, ps, ps)
    T = OFFSET + int(starts[-1]) + AFTER
    k, v = (torch.from_numpy(rng.standard_normal((T, 2, 128))).to(torch.float16).cuda() for _ in range(2))
    mine = slice(OFFSET, T - AFTER)
    want, cache = to_gpu(pool), to_gpu(pool)
    mdss.cache_append(want, 0, k[mine], v[mine], ids(starts), ids(table), ids(lengths))
    mdss.cache_append(cache, 0, k, v, ids(starts + OFFSET), ids(table), ids(lengths))
    same_pool(cache, to_pool(want))
