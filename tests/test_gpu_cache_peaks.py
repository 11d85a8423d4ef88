"""Attention rows that one token leads by far while its values vanish, so that the output is what the others add up to.

The bound is that of tests/test_gpu_cache_attention.py: a rounding of the weights to 11 bits, 2^-11 of sum p |v| in each element,
however small the weights are beside the largest.  What the products' fp32 sums lose beside a zero is nothing."""
import math

import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from cache_cases import ids, starts_of, tables, to_gpu
from oracle import cache as oc
from test_gpu_cache_attention import check

pytestmark = pytest.mark.gpu


def peaked(rng, kind, d, ps, new, lengths, group, lead, flat, leaders, ve=None):
    """A pool and queries of equal rows: the key of each leading token scores `lead` nats above the others' (which score within
    1 where not flat), its values are 0; the others' are positive, or all equal."""
    pages = sum((x + ps - 1) // ps for x in lengths)
    pool = oc.new_pool(1, pages, 1, d, ps)
    table = tables(lengths, ps, pages, rng, extra=0)
    for s, L in enumerate(lengths):
        k = np.zeros((L, d))
        if not flat:
            k[:, 1] = rng.uniform(-1.0, 1.0, L)
        v = np.ones((L, d)) if flat else rng.uniform(0.25, 4.0, (L, d))
        for at in leaders:
            if at < L:
                k[at], v[at] = 0.0, 0.0
                k[at, 0] = 1.0
        for j in range((L + ps - 1) // ps):
            page, m = table[s, j], min(ps, L - j * ps)
            for name, x, e in (("k", k, -8), ("v", v, -6 if ve is None else int(ve[j % len(ve)]))):
                codes = np.zeros((ps, d), np.uint8)
                codes[:m] = oc.encode(x[j * ps:j * ps + m] * 2.0 ** (8 if name == "k" else 6))
                oc.put_tokens(pool, name, 0, page, 0, codes)
                pool[name + "_exp"][0, page, 0] = e
    q = torch.zeros((sum(new), group, d), dtype=torch.float32)
    q[..., 0], q[..., 1] = lead, 1.0
    q = q.to(torch.bfloat16 if kind == "bf16" else torch.float16)
    return pool, table, q.cuda(), q.double().numpy()


def run(pool, table, q, q64, new, lengths, kind, d, **hints):
    cache, starts, table_, lengths_ = to_gpu(pool), ids(starts_of(new)), ids(table), ids(lengths)
    out, lse = mdss.cache_attention(q, cache, 0, starts, table_, lengths_, scale=1.0, want_lse=True, **hints)
    torch.cuda.synchronize()
    # rows of one token are equal: the oracle takes the first query head
    want = oc.attention(pool, 0, q64[:, :1], starts_of(new), table, lengths, 1.0)
    for g in range(q64.shape[1]):
        check(out[:, g:g + 1], lse[:, g:g + 1], want, kind, d, max(lengths))


LEADS = [9.0, 12.0, 14.0, 16.0, 17.5, 20.0, 24.0, 30.0]


@pytest.mark.parametrize("flat", [True, False])
@pytest.mark.parametrize("lead", LEADS)
@pytest.mark.parametrize("new,group", [([1], 2), ([5], 8), ([3], 8), ([70], 2)])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_a_leading_token_without_values(d, new, group, lead, flat):
    """One, two and four row tiles of few rows and many rows; the first token leads, or one inside a tile."""
    rng = np.random.default_rng([d, new[0], group, int(lead * 2), flat])
    lengths = [1500]
    for leaders in ((0,), (777,)):
        case = peaked(rng, "bf16", d, 64, new, lengths, group, lead, flat, leaders)
        run(*case, new, lengths, "bf16", d)


@pytest.mark.parametrize("length", [1, 2, 5, 17, 64, 65, 130])
@pytest.mark.parametrize("lead", [12.0, 17.5, 24.0])
@pytest.mark.parametrize("group", [1, 80])
def test_short_sequences(length, lead, group):
    rng = np.random.default_rng([length, int(lead), group])
    case = peaked(rng, "bf16", 64, 16, [1], [length], group, lead, True, (0,))
    run(*case, [1], [length], "bf16", 64)


@pytest.mark.parametrize("new,group", [([1], 8), ([4], 8), ([40], 4)])
@pytest.mark.parametrize("length", [32768, 131072])
def test_long_sequences(length, new, group):
    """0.999 of the weight on a token without values, the rest spread over the sequence: whole and in splits."""
    rng = np.random.default_rng([length, new[0]])
    lead = math.log(999.0 * length)
    case = peaked(rng, "bf16", 64, 256, new, [length], group, lead, False, (0,))
    run(*case, new, [length], "bf16", 64)
    run(*case, new, [length], "bf16", 64, max_length=1)  # a hint that leaves the whole sequence to one workgroup


@pytest.mark.parametrize("new,group", [([2], 4), ([70], 2)])
@pytest.mark.parametrize("ve", [(0, -30), (-40, 40), (40, -40), (-40, 0, -20), (8, -12, -30, -6)])
def test_pages_of_unlike_scale_under_a_leader(new, group, ve):
    """A page's exponent shifts its weights as a lead does; where the page of larger scale holds nothing in an element, the
    others' terms are that element."""
    rng = np.random.default_rng([new[0], len(ve), ve[0] + 40])
    lengths = [400]
    pool, table, q, q64 = peaked(rng, "bf16", 64, 16, new, lengths, group, 6.0, False, (3,), ve)
    v = pool["v"]
    large = pool["v_exp"][0, table[0], 0] == max(ve)
    v[0, table[0][large], 0, :, ::2] = 0
    run(pool, table, q, q64, new, lengths, "bf16", 64)


@pytest.mark.parametrize("new,group", [([1], 1), ([70], 1)])
def test_leaders_behind_each_other(new, group):
    """The maximum grows along the sequence, by more and by less than what the sums are rescaled for."""
    rng = np.random.default_rng([5, new[0]])
    lengths, d, ps = [900], 64, 16
    pool, table, q, q64 = peaked(rng, "bf16", d, ps, new, lengths, group, 0.0, False, ())
    for i, at in enumerate((5, 100, 101, 300, 301, 640)):
        codes = oc.tokens_of(pool, "k", 0, table[0, at // ps], 0).copy()
        codes[at % ps] = 0
        codes[at % ps, 2] = oc.encode(np.array([(0.5 + i) * 0.25 * 2.0 ** 8]))[0]
        oc.put_tokens(pool, "k", 0, table[0, at // ps], 0, codes)
        values = oc.tokens_of(pool, "v", 0, table[0, at // ps], 0).copy()
        values[at % ps] = 0
        oc.put_tokens(pool, "v", 0, table[0, at // ps], 0, values)
    for step in (8.0, 16.0, 24.0):
        q[..., 2] = step
        q64 = q.double().cpu().numpy()
        run(pool, table, q, q64, new, lengths, "bf16", d)
