"""Attention over rows that lack pages in a pool whose page 0 is free and holds any bytes, exponents out of their range among
them: what stands in for a missing page is never seen.  Bound: tests/test_gpu_cache_attention.py's."""
import numpy as np
import pytest

from cache_cases import tables
from oracle import cache as oc
from test_gpu_cache_attention import fill, queries, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponent", [-128, -127, -90, 88, 127])
@pytest.mark.parametrize("new,group", [([1, 1], 1), ([1, 1], 24), ([5, 6], 8), ([70, 40], 2)])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_page_0_holds_anything(d, new, group, exponent):
    rng = np.random.default_rng([d, new[0], group, exponent + 128])
    ps, lengths, pages = 16, [300, 210], 40
    pool = oc.new_pool(1, pages, 1, d, ps)
    fill(pool, rng)
    table = tables(lengths, ps, pages - 1, rng) + 1  # page 0 is nobody's
    table[table == 0] = -1
    for n in ("k", "v"):
        pool[n][0, 0] = 0x7f
        pool[n + "_exp"][0, 0] = exponent
    table[0, [0, 5, 9]] = [-1, -7, 1000]  # pages that are missing or none of the pool's
    table[1, 3] = pages
    q, q64 = queries(rng, (sum(new), group, d), "bf16")
    run(pool, q, q64, new, lengths, table, "bf16")
