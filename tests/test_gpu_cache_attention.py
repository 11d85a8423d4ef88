"""Attention over the paged 8-bit cache against oracle/cache.py.

The bound on an output element: weights rounded to f16 (2^-11 of sum p |v|); scores off by their fp32 sums (D terms,
2^-24 of sum |q| |k| each) and by t's rounding (2^-24 of |s| log2 e + 40), twice since the normaliser takes
part; fp32 sums over the tokens (2^-24 a token); the output's own rounding (half a unit: 2^-8 of it for bf16's 8 bits, 2^-11
for f16's 11, with 2^-25 below f16's normal range)."""
import math

import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from cache_cases import TYPES, ids, starts_of, tables, to_gpu
from oracle import cache as oc

pytestmark = pytest.mark.gpu


def fill(pool, rng, lo=-7, hi=-4):
    """Normal codes and exponents of a few octaves everywhere."""
    for n in ("k", "v"):
        pool[n][...] = oc.encode(rng.standard_normal(pool[n].shape) * 60.0)
        pool[n + "_exp"][...] = rng.integers(lo, hi, pool[n + "_exp"].shape)


def queries(rng, shape, kind):
    t = torch.from_numpy(rng.standard_normal(shape)).to(TYPES[kind])
    return t.cuda(), t.double().numpy()


def check(out, lse, want, kind, d, tokens):
    ref, rlse, mag, slack = want
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    score = 2.0 * (d * 2.0 ** -24 * slack + 2.0 ** -24 * (1.5 * slack + 40.0))[..., None]
    tol = mag * (2.0 ** -11 + score + (tokens + 64) * 2.0 ** -24) * 1.01
    tol = tol + np.abs(ref) * (2.0 ** -8 if kind == "bf16" else 2.0 ** -11) * 1.01 + (2.0 ** -25 if kind == "f16" else 1e-38)
    assert np.array_equal(np.isnan(out), np.isnan(ref))
    bad = ~(np.abs(out - ref) <= tol) & ~np.isnan(ref)
    assert not bad.any(), f"{bad.sum()} elements, worst {np.nanmax(np.abs(out - ref) / tol):.3g} of the bound"
    fine = np.isfinite(rlse)
    assert np.array_equal(np.isneginf(rlse), np.isneginf(lse)) and np.array_equal(np.isnan(rlse), np.isnan(lse))
    ltol = score[..., 0] + (tokens + 64) * 2.0 ** -24 + 2.0 ** -22 * (np.abs(rlse) + 30.0)
    assert np.all(np.abs(lse - rlse)[fine] <= ltol[fine])


def run(pool, q, q64, new, lengths, table, kind, scale=None, uniform=False, layer=0, **hints):
    d = q64.shape[2]
    out, lse = mdss.cache_attention(q, to_gpu(pool), layer, None if uniform else ids(starts_of(new)), ids(table),
                                    ids(lengths), scale=scale, want_lse=True, **hints)
    torch.cuda.synchronize()
    want = oc.attention(pool, layer, q64, starts_of(new), table, lengths, 1 / math.sqrt(d) if scale is None else scale)
    check(out, lse, want, kind, d, max(lengths))
    return out


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("d,ps,heads,group", [(64, 16, 2, 1), (64, 64, 1, 8), (96, 32, 2, 3), (96, 16, 1, 16),
                                               (128, 16, 2, 4), (128, 128, 1, 5), (128, 64, 8, 2), (256, 32, 1, 2),
                                               (256, 256, 2, 8)])
def test_ragged_batches(d, ps, heads, group, kind):
    rng = np.random.default_rng([d, ps, heads, group])
    new = [1, 0, 3, 1, 9, 2]
    lengths = [1, 30, 3, 257, 64, 700]
    pages = sum((x + ps - 1) // ps for x in lengths) + 2
    pool = oc.new_pool(2, pages, heads, d, ps)
    fill(pool, rng)
    q, q64 = queries(rng, (sum(new), heads * group, d), kind)
    run(pool, q, q64, new, lengths, tables(lengths, ps, pages, rng), kind, layer=1)


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 255, 256, 257, 1000])
def test_lengths_of_one_token(length):
    rng = np.random.default_rng(length)
    ps = 32
    lengths = [length, max(1, length - 1), length + 1]
    pages = sum((x + ps - 1) // ps for x in lengths)
    pool = oc.new_pool(1, pages, 1, 64, ps)
    fill(pool, rng)
    q, q64 = queries(rng, (3, 4, 64), "bf16")
    run(pool, q, q64, [1, 1, 1], lengths, tables(lengths, ps, pages, rng), "bf16", uniform=True)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n,group", [(7, 2), (8, 2), (30, 1), (33, 1), (16, 4), (70, 2), (130, 1), (40, 8)])
def test_many_rows(n, group, d):
    """Row tiles of every size: rows that share the tokens and rows that do not, prompts without a past."""
    rng = np.random.default_rng([n, group, d])
    ps = 16
    new, lengths = [n, n - 1, n], [n, n + 150, n + 3]
    pages = sum((x + ps - 1) // ps for x in lengths)
    pool = oc.new_pool(1, pages, 1, d, ps)
    fill(pool, rng)
    q, q64 = queries(rng, (sum(new), group, d), "f16")
    table = tables(lengths, ps, pages, rng)
    run(pool, q, q64, new, lengths, table, "f16")
    run(pool, q, q64, new, lengths, table, "f16", max_new=n, max_length=max(lengths))
    run(pool, q, q64, new, lengths, table, "f16", max_new=1, max_length=1)  # hints choose no token
    run(pool, q[:2 * n], q64[:2 * n], [n, n], [n, n + 150], table[:2], "f16", uniform=True)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_split_over_a_long_sequence(kind):
    rng = np.random.default_rng(11)
    ps, lengths = 64, [9000, 40, 4097]
    pages = sum((x + ps - 1) // ps for x in lengths)
    pool = oc.new_pool(1, pages, 2, 128, ps)
    fill(pool, rng)
    table = tables(lengths, ps, pages, rng)
    q, q64 = queries(rng, (3, 8, 128), kind)
    run(pool, q, q64, [1, 1, 1], lengths, table, kind, uniform=True)
    run(pool, q, q64, [1, 1, 1], lengths, table, kind, uniform=True, max_length=5000)
    q, q64 = queries(rng, (60, 8, 128), kind)  # (rows that do not share a wave, split too)
    run(pool, q, q64, [20, 10, 30], lengths, table, kind)


def test_bytes_past_the_tokens_are_never_seen():
    """Any bytes, NaN codes and extreme exponents among them, in what is not a sequence's."""
    rng = np.random.default_rng(12)
    ps, lengths, new = 32, [5, 33, 100, 1], [2, 33, 1, 1]
    pages = 12
    pool = oc.new_pool(1, pages, 2, 64, ps, rng)
    table = tables(lengths, ps, pages, rng)
    for s, L in enumerate(lengths):
        for j in range((L + ps - 1) // ps):
            m = min(ps, L - j * ps)
            for h in range(2):
                for n in ("k", "v"):
                    codes = oc.tokens_of(pool, n, 0, table[s, j], h).copy()
                    codes[:m] = oc.encode(rng.standard_normal((m, 64)) * 60)
                    codes[m:] = 0x7f
                    oc.put_tokens(pool, n, 0, table[s, j], h, codes)
                    pool[n + "_exp"][0, table[s, j], h] = -6
    q, q64 = queries(rng, (sum(new), 4, 64), "bf16")
    assert torch.isfinite(run(pool, q, q64, new, lengths, table, "bf16")).all()


@pytest.mark.parametrize("new", [[1, 1], [6, 3], [70, 40]])
def test_nan_reaches_only_the_rows_that_see_it(new):
    rng = np.random.default_rng([13] + new)
    ps, lengths = 16, [100, 90]
    pages = 14
    pool = oc.new_pool(1, pages, 1, 64, ps)
    fill(pool, rng)
    table = tables(lengths, ps, pages, rng)

    def spoil(name, s, token, element):
        codes = oc.tokens_of(pool, name, 0, table[s, token // ps], 0).copy()
        codes[token % ps, element] = 0xff
        oc.put_tokens(pool, name, 0, table[s, token // ps], 0, codes)

    spoil("v", 0, 98, 5)   # seen by the last two rows, in one element
    spoil("v", 0, 97, 63)
    spoil("k", 1, 88, 0)   # seen by the last two rows, in all
    q, q64 = queries(rng, (sum(new), 4, 64), "f16")
    run(pool, q, q64, new, lengths, table, "f16")


def test_rows_that_see_nothing():
    """No tokens, fewer tokens than queries, pages that are missing."""
    rng = np.random.default_rng(14)
    ps = 16
    new, lengths = [1, 3, 2, 4, 2], [0, 1, 40, 2, 35]
    pool = oc.new_pool(1, 12, 1, 64, ps)
    fill(pool, rng)
    table = np.array([[-1] * 3, [0, -1, -1], [-1, 3, 1000], [7, -1, -1], [-1, -1, -1]], np.int32)
    q, q64 = queries(rng, (sum(new), 2, 64), "bf16")
    run(pool, q, q64, new, lengths, table, "bf16")


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_pages_of_unlike_scale(kind):
    """Exponents over the whole range: tokens of tiny values keep their part of the normaliser, and a page of large
    values that has no weight takes nothing from the others."""
    rng = np.random.default_rng(15)
    ps, lengths = 16, [400, 64]
    pages = 30
    pool = oc.new_pool(1, pages, 1, 64, ps)
    fill(pool, rng)
    pool["v_exp"][...] = rng.choice([-40, -20, -6, 0, 8], pool["v_exp"].shape)
    table = tables(lengths, ps, pages, rng)
    q, q64 = queries(rng, (2, 2, 64), kind)
    run(pool, q, q64, [1, 1], lengths, table, kind, uniform=True)
    pool["v"][:, table[1, 0]] = 0  # a page of zeros at the smallest exponent
    pool["v_exp"][:, table[1, 0]] = -40
    pool["v_exp"][:, table[1, 1]] = 8
    run(pool, q, q64, [1, 1], lengths, table, kind, uniform=True)


def test_strided_queries_scale_and_output():
    rng = np.random.default_rng(16)
    ps, new, lengths = 16, [2, 1], [50, 20]
    pool = oc.new_pool(1, 8, 2, 64, ps)
    fill(pool, rng)
    table = tables(lengths, ps, 8, rng)
    wide, wide64 = queries(rng, (3, 8, 64), "bf16")
    run(pool, wide[:, 2:6], wide64[:, 2:6], new, lengths, table, "bf16", scale=0.3)
    run(pool, wide[:, 4:], wide64[:, 4:], new, lengths, table, "bf16", scale=-0.2)
    odd = torch.zeros(wide.numel() + 3, dtype=torch.bfloat16, device="cuda:0")
    odd[3:] = wide.reshape(-1)
    out = torch.empty((3, 8, 64), dtype=torch.bfloat16, device="cuda:0")
    got = run(pool, odd[3:].view(3, 8, 64), wide64, new, lengths, table, "bf16", out=out)
    assert got.data_ptr() == out.data_ptr()


def test_large_and_infinite_scores():
    rng = np.random.default_rng(17)
    ps, lengths = 16, [40, 70]
    pool = oc.new_pool(1, 10, 1, 64, ps)
    fill(pool, rng)
    pool["k_exp"][...] = 3  # scores in the hundreds: one token takes all
    table = tables(lengths, ps, 10, rng)
    q, q64 = queries(rng, (2, 1, 64), "bf16")
    run(pool, q, q64, [1, 1], lengths, table, "bf16", uniform=True, scale=0.02)
    q[0, 0, 0] = float("nan")
    q64[0, 0, 0] = math.nan
    run(pool, q, q64, [1, 1], lengths, table, "bf16", uniform=True, scale=0.02)


def test_another_stream_and_a_graph():
    rng = np.random.default_rng(18)
    ps, lengths = 16, [3000, 700]
    pages = 300
    pool = oc.new_pool(1, pages, 2, 64, ps)
    fill(pool, rng)
    cache = to_gpu(pool)
    table, length = ids(tables(lengths, ps, pages, rng)), ids(lengths)
    q, _ = queries(rng, (2, 8, 64), "bf16")
    torch.cuda.synchronize()
    want = mdss.cache_attention(q, cache, 0, None, table, length)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = mdss.cache_attention(q, cache, 0, None, table, length)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = mdss.cache_attention(q, cache, 0, None, table, length)
    for _ in range(3):
        got.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        torch.randn(1000, device="cuda:0").sum().item()
