"""Attention where scores are finite and huge: the softmax of scores that lie apart by far more than their own rounding is 1 for the
largest, and equal scores share it, whatever the scales of their pages.  Keys have one element and factors are small whole
numbers times powers of two, so scores are exact and the outputs known."""
import math

import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from cache_cases import ids, tables, to_gpu
from oracle import cache as oc

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 500), (3, 8, 500), (5, 8, 500), (70, 2, 500), (1, 4, 9000), (40, 4, 9000)]  # new tokens, group, length


def setup(d, ps, length, codes, rng):
    """One sequence: `codes` (token -> key code value, ke) over keys of -448 at the exponent 0, values 1 .. 7."""
    pages = (length + ps - 1) // ps
    pool = oc.new_pool(1, pages, 1, d, ps)
    table = tables([length], ps, pages, rng, extra=0)
    values = rng.integers(1, 8, (length, d)).astype(np.float64)
    for j in range(pages):
        m = min(ps, length - j * ps)
        key, ke, ve = np.zeros((ps, d)), 0, int(rng.integers(-6, 5))
        key[:m, 0] = -1.0
        for t, (code, e) in codes.items():
            if t // ps == j:
                key[t % ps, 0], ke = code, e
        v = np.zeros((ps, d))
        v[:m] = values[j * ps:j * ps + m] * 2.0 ** -ve
        oc.put_tokens(pool, "k", 0, table[0, j], 0, oc.encode(key))
        oc.put_tokens(pool, "v", 0, table[0, j], 0, oc.encode(v))
        pool["k_exp"][0, table[0, j], 0], pool["v_exp"][0, table[0, j], 0] = ke, ve
    return pool, table, values


def attend(pool, table, length, n, group, d, power, sign):
    q = torch.zeros((n, group, d), dtype=torch.bfloat16, device="cuda:0")
    q[..., 0] = sign * 2.0 ** power
    out, lse = mdss.cache_attention(q, to_gpu(pool), 0, None, ids(table), ids([length]), scale=1.0, want_lse=True)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


@pytest.mark.parametrize("n,group,length", SHAPES)
@pytest.mark.parametrize("power", [0, 6, 9, 12, 16, 18, 20, 21, 22, 23, 24, 26, 28, 30, 40, 60])
def test_one_leads(n, group, length, power):
    """Scores of 320 2^power and below 0; then all below 0, of which the least by far is the largest."""
    rng = np.random.default_rng([power, n, length])
    at = length - n - 3  # seen by every row
    for sign, code in ((1.0, 320.0), (-1.0, -5.0)):
        codes = {at: (code, 0)}
        if sign < 0:
            codes = {at: (0.625, 0)}
        pool, table, values = setup(64, 16, length, codes, rng)
        if sign < 0:  # every other key 448: scores of -448 2^power beside -0.625 2^power
            for j in range(table.shape[1]):
                k = oc.tokens_of(pool, "k", 0, table[0, j], 0).copy()
                x = oc.decode(k)
                x[x == -1.0] = 448.0
                oc.put_tokens(pool, "k", 0, table[0, j], 0, oc.encode(x))
        out, lse = attend(pool, table, length, n, group, 64, power, sign)
        score = (320.0 if sign > 0 else -0.625) * 2.0 ** power
        np.testing.assert_array_equal(out, np.broadcast_to(values[at], out.shape))
        # (one multiplication by log2 e, one back: 2^-22 of the score; nothing is added below 1e-38)
        assert np.all(np.abs(lse - score) <= 2.0 ** -22 * abs(score) + 2.0 ** -20)


@pytest.mark.parametrize("n,group,length", SHAPES)
@pytest.mark.parametrize("power", [0, 9, 12, 14, 16, 20, 22, 24, 28, 40, 60])
def test_equal_scores_share(n, group, length, power):
    """Three equal scores in pages of unlike key and value exponents, in one tile of 64 tokens and far apart."""
    rng = np.random.default_rng([power, n, length, 1])
    where = [2, 20, length - n - 3]
    pool, table, values = setup(64, 16, length, {where[0]: (64.0, 0), where[1]: (32.0, 1), where[2]: (256.0, -2)}, rng)
    for t, e in ((where[1], 1), (where[2], -2)):  # the other keys of a page keep their scores below 0
        k = oc.tokens_of(pool, "k", 0, table[0, t // 16], 0).copy()
        assert (oc.decode(k)[:, 0] > 0).sum() == 1
    out, lse = attend(pool, table, length, n, group, 64, power, 1.0)
    want = values[where].mean(axis=0)
    # the output's rounding to bf16 (2^-9 of it), and three weights equal but for theirs
    assert np.all(np.abs(out - want) <= 2.0 ** -8 * want)
    score = 64.0 * 2.0 ** power
    assert np.all(np.abs(lse - (score + math.log(3.0))) <= 2.0 ** -22 * score + 2.0 ** -20)
