"""Pins of the rotary and shared-prefix counterparts."""
import math

import numpy as np

from oracle import cache as oc
from oracle import rotary as orot


def test_scores_depend_on_the_distance_alone():
    rng = np.random.default_rng(0)
    freq = orot.frequencies(32)
    q, k = rng.standard_normal((2, 1, 1, 40))
    for interleaved in (False, True):
        at = lambda a, b: (orot.rotate(q, freq, [a], interleaved) * orot.rotate(k, freq, [b], interleaved)).sum()  # noqa: E731
        assert abs(at(5, 2) - at(1003, 1000)) < 1e-9 and abs(at(5, 2) - at(5, 3)) > 1e-3
        assert abs(at(7, 7) - (q * k).sum()) < 1e-12


def test_one_pair_by_hand():
    x = np.array([[[3.0, 4.0, 9.0]]])
    got = orot.rotate(x, np.array([math.pi / 2]), [1], magnitude=2.0)
    np.testing.assert_allclose(got, [[[-8.0, 6.0, 9.0]]], atol=1e-12)
    np.testing.assert_allclose(orot.rotate(x, np.array([math.pi / 2]), [1], inverse=True), [[[4.0, -3.0, 9.0]]], atol=1e-12)
    wide = np.arange(1.0, 5.0)[None, None]
    f = np.array([math.pi, math.pi / 2])
    np.testing.assert_allclose(orot.rotate(wide, f, [1]), [[[-1, -4, -3, 2]]], atol=1e-12)
    np.testing.assert_allclose(orot.rotate(wide, f, [1], interleaved=True), [[[-1, -2, -4, 3]]], atol=1e-12)


def test_frequencies():
    np.testing.assert_allclose(orot.frequencies(8), [1, 0.1, 0.01, 0.001])
    np.testing.assert_allclose(orot.frequencies(8, scale=4.0), [0.25, 0.025, 0.0025, 0.00025])
    f = orot.frequencies(64, scale=8.0, original=4096)
    plain = orot.frequencies(64)
    turns = 4096 * plain / (2 * math.pi)
    assert (f[turns > 32] == plain[turns > 32]).all() and np.allclose(f[turns < 1], plain[turns < 1] / 8)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and ((f < plain) & (f > plain / 8))[mid].all()


def test_the_bound_holds():
    rng = np.random.default_rng(1)
    k = rng.standard_normal((50, 3, 24))
    freq = orot.frequencies(16)
    turned = orot.rotate(k, freq, rng.integers(0, 10 ** 6, 50), magnitude=1.3)
    assert (np.abs(turned).max(axis=2) <= orot.key_limit(k, 8, 1.3) * (1 + 1e-6)).all()


def test_shared_by_hand():
    table = np.array([[5, 6, 7, 8, 1], [5, 6, 7, 8, 2], [5, 6, 7, 8, 3], [-1] * 5, [5, 9, 7, 8, 4]], np.int32)
    lengths, starts = [70, 80, 66, 0, 70], np.arange(6)
    tokens, rows = oc.shared(10, 16, starts, table, lengths, [0, 4, 5])
    assert tokens.tolist() == [64, 64, 64, 0, 0] and rows.tolist() == [[0, 4, 0, 64], [4, 1, 4, 0]]
    assert oc.shared(10, 16, starts, table, lengths, [0, 5])[0].tolist() == [0] * 5  # page 9 in place of 6: 16 tokens are less than 64
    assert oc.shared(10, 16, starts, table, lengths, [0, 4], 65)[1].tolist() == [[0, 4, 0, 0]]
    assert oc.shared(10, 16, starts, table, lengths, [0, 4], 68)[0].tolist() == [0] * 5  # rows 0 and 1 alone, 64 of them
    assert oc.shared(7, 16, starts, table, lengths, [0, 4])[1][0].tolist() == [0, 4, 0, 0]  # (ids from 7 on are outside the pool)
