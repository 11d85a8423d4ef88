"""Pins of oracle/cache.py and oracle/beam.py: codes against torch's own e4m3 type, attention and the beam step against
dense torch in 64 bits, pages against what a search may hold."""
import math

import numpy as np
import pytest
import torch

from oracle import beam as ob
from oracle import cache as oc


def test_codes_are_the_types():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(oc.decode(codes), want)
    fine = ~np.isnan(want)
    np.testing.assert_array_equal(oc.encode(want[fine]), codes[fine])
    rng = np.random.default_rng(1)
    x = np.concatenate((rng.standard_normal(20000) * np.exp2(rng.integers(-12, 8, 20000)), [448.0, -448.0, 0.0, -0.0]))
    x = np.clip(x, -448, 448).astype(np.float32)
    mid = (want[fine][:-1] + want[fine][1:]) / 2  # halfway between neighbours: ties
    for v in (x, mid.astype(np.float32)):
        got = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        np.testing.assert_array_equal(oc.encode(v), got)
    assert oc.encode(np.array([1e9, -1e9, math.inf, -math.inf])).tolist() == [126, 254, 127, 255]


@pytest.mark.parametrize("a,e", [(0.0, -40), (448.0, 0), (448.1, 1), (447.9, 0), (1.0, -8), (1.75, -8), (1.76, -7), (1e-30, -40), (1e30, 40)])
def test_exponents(a, e):
    assert oc.exponent(a) == e


def test_append_reads_back():
    """What comes back is within half a step of what went in, relative to the page's largest value."""
    rng = np.random.default_rng(2)
    pool = oc.new_pool(1, 4, 2, 64, 16, rng)
    table = np.array([[2, 0], [3, -1]], np.int32)
    x = rng.standard_normal((30, 2, 64))
    starts = np.array([0, 20, 30])
    assert oc.append(pool, 0, x, -x, starts, table, [20, 10]) == set()
    for s, (a, b) in enumerate(((0, 20), (20, 30))):
        for h in range(2):
            k, ok = oc.sequence(pool, "k", 0, table[s], b - a, h)
            v, _ = oc.sequence(pool, "v", 0, table[s], b - a, h)
            assert ok.all()
            np.testing.assert_allclose(k, x[a:b, h], rtol=2.0 ** -4, atol=2.0 ** -9 * 2.0 ** -6)
            np.testing.assert_array_equal(k, -v)
    assert oc.append(pool, 0, x, x, starts, table, [40, 10]) == {0}


def test_attention_is_the_softmax():
    rng = np.random.default_rng(3)
    pool = oc.new_pool(1, 4, 2, 64, 16)
    for n in ("k", "v"):
        pool[n][...] = oc.encode(rng.standard_normal(pool[n].shape) * 50)
        pool[n + "_exp"][...] = -6
    table = np.array([[1, 3, 0]], np.int32)
    q = rng.standard_normal((3, 4, 64))
    out, lse, mag, slack = oc.attention(pool, 0, q, [0, 3], table, [40], 0.125)
    for hq in range(4):
        k = torch.from_numpy(oc.sequence(pool, "k", 0, table[0], 40, hq // 2)[0])
        v = torch.from_numpy(oc.sequence(pool, "v", 0, table[0], 40, hq // 2)[0])
        s = torch.from_numpy(q[:, hq]) @ k.T * 0.125
        s = s.masked_fill(torch.arange(40) > torch.arange(37, 40)[:, None], -math.inf)
        np.testing.assert_allclose(out[:, hq], (torch.softmax(s, 1) @ v).numpy(), rtol=1e-12, atol=1e-13)
        np.testing.assert_allclose(lse[:, hq], torch.logsumexp(s, 1).numpy(), rtol=1e-13)
    assert np.all(mag >= np.abs(out) - 1e-12) and slack.shape == (3, 4)


@pytest.mark.parametrize("seed", range(6))
def test_forks_keep_every_token(seed):
    """Whatever the parents: rows read what their parents read, a page that a row grows on is its own, and the counts are
    the rows'."""
    rng = np.random.default_rng([4, seed])
    ps, pages = 16, 60
    pool = oc.new_pool(2, pages, 1, 64, ps, rng)
    lengths = [20, 33, 16, 0]
    table = np.full((4, 6), -1, np.int32)
    order = iter(rng.permutation(pages))
    for s, L in enumerate(lengths):
        for j in range((L + ps - 1) // ps):
            table[s, j] = next(order)
    refs = np.zeros(pages, np.int32)
    refs[table[table >= 0]] = 1
    for _ in range(5):
        n = len(lengths)
        parent = rng.integers(-1, n, 5)
        keep = rng.integers(0, 60, 5)
        grow = rng.integers(0, 20, 5)
        before = {n: x.copy() for n, x in pool.items()}
        t, L, r, flagged = oc.fork(pool, table, lengths, refs, parent, keep, grow)
        held = np.zeros(pages, np.int32)
        for i, p in enumerate(parent):
            have = 0 if p < 0 else min(lengths[p], keep[i])
            for j in range((L[i] + ps - 1) // ps):
                held[t[i, j]] += 1
            for l in range(2):
                for j in range((have + ps - 1) // ps):
                    for n in ("k", "v", "k_exp", "v_exp"):
                        np.testing.assert_array_equal(pool[n][l, t[i, j]], before[n][l, table[p, j]])
            if L[i] > have and have % ps:
                assert r[t[i, have // ps]] == 1
        np.testing.assert_array_equal(held, r)
        assert not flagged
        table, lengths, refs = t, [int(x) for x in L], r


def test_compact_keeps_every_page():
    rng = np.random.default_rng(5)
    pool = oc.new_pool(1, 30, 1, 64, 16, rng)
    table = np.array([[29, 3, -1], [0, 17, 25]], np.int32)
    refs = np.zeros(30, np.int32)
    refs[[29, 3, 0, 17, 25]] = [2, 1, 1, 1, 3]
    before = {n: x.copy() for n, x in pool.items()}
    t, r, used = oc.compact(pool, table, [20, 48], refs)
    assert used == 5 and (r[5:] == 0).all() and sorted(t[t >= 0].tolist()) == [0, 1, 2, 3, 4]
    for a, b in zip(table[table >= 0], t[t >= 0]):
        assert refs[a] == r[b]
        for n in pool:
            np.testing.assert_array_equal(pool[n][:, b], before[n][:, a])
    assert t[0, 0] == 1 and t[1, 2] == 2 and t[1, 1] == 4  # the highest page to the lowest hole


def test_beam_is_the_flat_top():
    rng = np.random.default_rng(6)
    x = torch.from_numpy(rng.standard_normal((3, 4, 50)))
    s = torch.from_numpy(-rng.random((3, 4)))
    parent, token, score, done, refused = ob.select(x.numpy(), s.numpy(), eos=7)
    total = (torch.log_softmax(x, 2) + s[:, :, None]).view(3, -1)
    best = torch.topk(total, 4, dim=1)
    np.testing.assert_allclose(score, best.values.numpy(), rtol=1e-12)
    np.testing.assert_array_equal(parent * 50 + token, best.indices.numpy())
    assert not refused and np.array_equal(done, token == 7)
    state = rng.random((3, 4, 2))
    np.testing.assert_array_equal(ob.reorder(state, parent)[1, 2], state[1, parent[1, 2]])
