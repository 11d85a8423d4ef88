"""Attention over shared prefixes against oracle/cache.py's attention, which knows nothing of prefixes: the bound is that of
test_gpu_cache_attention.py (a row's parts are joined in fp32, as those of a split call are)."""
import math

import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from cache_cases import ids, to_gpu
from oracle import cache as oc
from shared_cases import Groups
from test_gpu_cache_attention import check, fill, queries

pytestmark = pytest.mark.gpu


def hints(c, tokens, rows):
    return dict(max_new=max(c.new), max_group=max(int(r[1]) for r in rows), max_shared=max(int(r[3]) for r in rows),
                max_own=max(L - int(t) for L, t in zip(c.lengths, tokens)))


def run(pool, c, q, q64, kind, scale=None, uniform=False, layer=0, least=0, cache=None, **kw):
    """Without hints and with them; returns the last result."""
    cache = to_gpu(pool) if cache is None else cache
    starts, table, lengths = None if uniform else ids(c.starts), ids(c.table), ids(c.lengths)
    shared = mdss.cache_shared(cache, c.T, starts, table, lengths, ids(c.groups), least=least)
    want = oc.attention(pool, layer, q64, c.starts, c.table, c.lengths, 1 / math.sqrt(q64.shape[2]) if scale is None else scale)
    for most in ({}, hints(c, shared[0].tolist(), shared[1].tolist())):
        out, lse = mdss.cache_attention_shared(q, cache, layer, starts, table, lengths, shared, scale=scale, want_lse=True, **most, **kw)
        torch.cuda.synchronize()
        check(out, lse, want, kind, q64.shape[2], max(c.lengths))
    return out


RAGGED = [(700, [(1, 30), (2, 5), (0, 7), (3, 300)]), (64, [(1, 1), (1, 2)]), (40, [(1, 9), (5, 70)]), (0, [(1, 1), (3, 3)]),
          (130, [(2, 2), (1, None), (2, 9)]), (300, [(4, 20)])]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("d,ps,heads,group", [(64, 16, 2, 1), (64, 64, 1, 8), (96, 32, 2, 3), (96, 16, 1, 16), (128, 16, 2, 4),
                                               (128, 128, 1, 5), (128, 64, 8, 2), (256, 32, 1, 2), (256, 256, 2, 8)])
def test_ragged_groups(d, ps, heads, group, kind):
    rng = np.random.default_rng([d, ps, heads, group])
    c = Groups(RAGGED, ps, rng)
    pool = oc.new_pool(2, c.pages, heads, d, ps)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, heads * group, d), kind)
    run(pool, c, q, q64, kind, layer=1)


@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("W,n,group", [(2, 1, 1), (16, 1, 1), (17, 1, 2), (16, 2, 2), (7, 3, 4), (33, 1, 4), (65, 1, 8), (3, 40, 2), (5, 1, 16)])
def test_rows_of_every_kernel(W, n, group, d):
    """Row tiles of 16, 32 and 64 shared by the waves, and waves of rows of their own, for the prefix and for what follows."""
    rng = np.random.default_rng([W, n, group, d])
    c = Groups([(1100, [(n, n + int(x)) for x in rng.integers(0, 200, W)]), (129, [(n, n + 3)] * W)], 16, rng)
    pool = oc.new_pool(1, c.pages, 1, d, 16)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, group, d), "f16")
    run(pool, c, q, q64, "f16", uniform=True)
    if d == 128:
        run(pool, c, q, q64, "f16")


@pytest.mark.parametrize("prefix", [63, 64, 65, 127, 128, 191, 192, 256, 1000, 4096])
def test_prefix_lengths(prefix):
    rng = np.random.default_rng(prefix)
    c = Groups([(prefix, [(1, 1 + i) for i in range(5)]), (prefix + 64, [(1, 1)] * 3)], 32, rng)
    pool = oc.new_pool(1, c.pages, 2, 64, 32)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, 4, 64), "bf16")
    run(pool, c, q, q64, "bf16", uniform=True)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_long_prefix_and_long_tails(kind):
    """Both parts split over workgroups, unevenly."""
    rng = np.random.default_rng(11)
    c = Groups([(9000, [(1, 3000), (1, 1), (1, 700)]), (200, [(1, 40), (1, 5000)])], 64, rng)
    pool = oc.new_pool(1, c.pages, 2, 128, 64)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, 8, 128), kind)
    run(pool, c, q, q64, kind, uniform=True)
    q, q64 = queries(rng, (c.T, 80, 128), kind)  # (40 rows a token: the waves take different ones)
    run(pool, c, q, q64, kind)


def test_rows_that_share_nothing():
    """Groups of one, rows in no group, rows shorter than `least`, and none at all."""
    rng = np.random.default_rng(12)
    c = Groups([(300, [(1, 20)]), (300, [(1, 20), (2, 30), (1, 90)]), (70, [(1, 1)] * 4)], 16, rng)
    pool = oc.new_pool(1, c.pages, 2, 64, 16)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, 4, 64), "bf16")
    for groups in (c.groups, [0], [1, 4], [0, 1, 2, 3, 4, 5, 6, 7, 8], [0, 8]):
        c.groups = groups
        starts, table, lengths = ids(c.starts), ids(c.table), ids(c.lengths)
        cache = to_gpu(pool)
        for least in (0, 200):
            shared = mdss.cache_shared(cache, c.T, starts, table, lengths, ids(groups), least=least)
            out, lse = mdss.cache_attention_shared(q, cache, 0, starts, table, lengths, shared, want_lse=True)
            check(out, lse, oc.attention(pool, 0, q64, c.starts, c.table, c.lengths, 0.125), "bf16", 64, 400)


def test_rows_that_see_nothing_and_tokens_of_no_sequence():
    rng = np.random.default_rng(13)
    c = Groups([(200, [(2, 9), (3, None), (1, 1), (1, 30)]), (500, [(1, None), (1, None)])], 16, rng)
    c.lengths[1] = 1  # three new tokens of which the last alone is there, and has no page
    pool = oc.new_pool(1, c.pages, 1, 64, 16)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T + 4, 2, 64), "f16")
    starts, table, lengths = ids(c.starts), ids(c.table), ids(c.lengths)
    cache = to_gpu(pool)
    shared = mdss.cache_shared(cache, c.T, starts, table, lengths, ids(c.groups))
    assert shared[0].tolist() == [192, 0, 192, 192, 0, 0]
    out = torch.full((c.T + 4, 2, 64), 5.0, dtype=torch.float16, device="cuda:0")
    _, lse = mdss.cache_attention_shared(q, cache, 0, starts, table, lengths, shared, want_lse=True, out=out)
    torch.cuda.synchronize()
    check(out[:c.T], lse[:c.T], oc.attention(pool, 0, q64[:c.T], c.starts, c.table, c.lengths, 0.125), "f16", 64, 600)
    assert bool((out[2:5] == 0).all()) and bool(torch.isinf(lse[2:5]).all()) and bool((out[c.T:] == 5.0).all())


def test_bytes_past_the_tokens_are_never_seen():
    """NaN codes and extreme exponents in the rest of pages and in pages of nobody, at the borders of prefix and own tokens."""
    rng = np.random.default_rng(14)
    ps = 32
    c = Groups([(64, [(1, 1), (1, 5), (2, 33)]), (90, [(1, 2), (3, 40)])], ps, rng)
    pool = oc.new_pool(1, c.pages, 2, 64, ps, rng)
    for s, L in enumerate(c.lengths):
        for j in range((L + ps - 1) // ps):
            m = min(ps, L - j * ps)
            for h in range(2):
                for n in ("k", "v"):
                    codes = oc.tokens_of(pool, n, 0, c.table[s, j], h).copy()
                    codes[:m] = oc.encode(rng.standard_normal((m, 64)) * 60)
                    codes[m:] = 0x7f
                    oc.put_tokens(pool, n, 0, c.table[s, j], h, codes)
                    pool[n + "_exp"][0, c.table[s, j], h] = -6
    q, q64 = queries(rng, (c.T, 4, 64), "bf16")
    assert torch.isfinite(run(pool, c, q, q64, "bf16")).all()


@pytest.mark.parametrize("group", [2, 40])
def test_nan_reaches_only_the_rows_that_see_it(group):
    """In the prefix: all rows of the group; in a sequence's own tokens: its rows from there on."""
    rng = np.random.default_rng([15, group])
    c = Groups([(128, [(3, 20), (2, 9)]), (128, [(2, 8), (1, 1)]), (70, [(1, 5), (1, 6)])], 16, rng)
    pool = oc.new_pool(1, c.pages, 1, 64, 16)
    fill(pool, rng)

    def spoil(name, s, token, element):
        codes = oc.tokens_of(pool, name, 0, c.table[s, token // 16], 0).copy()
        codes[token % 16, element] = 0xff
        oc.put_tokens(pool, name, 0, c.table[s, token // 16], 0, codes)

    spoil("v", 0, 100, 5)
    spoil("v", 0, 146, 9)   # (the second of its new tokens)
    spoil("k", 2, 135, 1)   # (the last of its new tokens)
    q, q64 = queries(rng, (c.T, group, 64), "f16")
    run(pool, c, q, q64, "f16")


def test_missing_pages():
    """A page that all rows lack ends what they share; one of a row's own is not seen."""
    rng = np.random.default_rng(16)
    c = Groups([(400, [(1, 40), (1, 20), (2, 90)])], 16, rng)
    c.table[:, 13] = c.pages + 3
    c.table[2, 27] = -1
    pool = oc.new_pool(1, c.pages, 2, 64, 16)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, 4, 64), "bf16")
    run(pool, c, q, q64, "bf16")


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_pages_of_unlike_scale_and_large_scores(kind):
    rng = np.random.default_rng(17)
    c = Groups([(320, [(1, 40), (1, 3), (1, 100)])], 16, rng)
    pool = oc.new_pool(1, c.pages, 1, 64, 16)
    fill(pool, rng)
    pool["v_exp"][...] = rng.choice([-40, -20, -6, 0, 8], pool["v_exp"].shape)
    q, q64 = queries(rng, (c.T, 2, 64), kind)
    run(pool, c, q, q64, kind, uniform=True)
    fill(pool, rng)
    pool["k_exp"][...] = 3  # one token takes all, in the prefix or past it
    run(pool, c, q, q64, kind, uniform=True, scale=0.02)
    pool["k_exp"][...] = 16  # scores of 2^20
    run(pool, c, q, q64, kind, uniform=True)


@pytest.mark.parametrize("group", [2, 40])
def test_queries_that_are_not_finite(group):
    """They spoil their own row alone, whichever part of it the kernels take first."""
    rng = np.random.default_rng([21, group])
    c = Groups([(300, [(1, 20), (2, 70)]), (128, [(1, 1)] * 3)], 16, rng)
    pool = oc.new_pool(1, c.pages, 1, 64, 16)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, group, 64), "bf16")
    for t, hq, value in ((0, 1, math.nan), (2, 0, math.inf), (4, 1, -math.inf)):
        q[t, hq, 5], q64[t, hq, 5] = value, value
    out = run(pool, c, q, q64, "bf16")
    assert sorted({tuple(x) for x in torch.nonzero(torch.isnan(out))[:, :2].tolist()}) == [(0, 1), (2, 0), (4, 1)]


@pytest.mark.parametrize("G,W,n,heads,group,d,prefix", [(5, 8, 1, 8, 2, 64, 3000), (5, 8, 1, 8, 8, 128, 3000), (4, 6, 2, 8, 1, 96, 5000), (2, 3, 1, 8, 4, 256, 20000),
                                                        (2, 40, 1, 8, 2, 64, 5100), (2, 40, 1, 8, 4, 128, 5100), (1, 10, 4, 8, 1, 128, 12000)])
def test_calls_that_are_large_enough_to_go_together(G, W, n, heads, group, d, prefix):
    """With every hint, so that prefixes and own tokens are cut as a program's are, by each kernel."""
    rng = np.random.default_rng([G, W, n, group, d])
    c = Groups([(prefix - 700 * g, [(n, n + int(x)) for x in rng.integers(0, 90, W)]) for g in range(G)], 64, rng)
    pool = oc.new_pool(1, c.pages, heads, d, 64)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, heads * group, d), "bf16")
    cache, starts, table, lengths = to_gpu(pool), ids(c.starts), ids(c.table), ids(c.lengths)
    shared = mdss.cache_shared(cache, c.T, starts, table, lengths, ids(c.groups))
    most = hints(c, shared[0].tolist(), shared[1].tolist())
    assert len(c.new) * heads * (most["max_shared"] // 64) >= (49152 if most["max_group"] * group > 64 else 12288)
    out, lse = mdss.cache_attention_shared(q, cache, 0, starts, table, lengths, shared, want_lse=True, **most)
    torch.cuda.synchronize()
    rows = rng.choice(len(c.new), 4, replace=False)  # (the oracle takes its time: some of the sequences)
    for s in rows:
        own = slice(c.starts[s], c.starts[s + 1])
        want = oc.attention(pool, 0, q64[own], [0, n], c.table[s:s + 1], c.lengths[s:s + 1], d ** -0.5)
        check(out[own], lse[own], want, "bf16", d, max(c.lengths))
    # The others against the call that knows no prefixes: both are within the bound of the same values, whose sums of p |v| are
    # attention over the values without their signs (2^-8 off at most itself).  Scores are off by 2 (d 2^-24 15 + 63 2^-24) < 2^-11
    # here, since |scale| |q| . |k| is below 15 (256 elements of 1 and 4 at most in q, of some 1 in k, times 1/16).
    plain, plse = mdss.cache_attention(q, cache, 0, starts, table, lengths, want_lse=True)
    mag = mdss.cache_attention(q, mdss.PagedCache(cache.k, cache.v & 127, cache.k_exp, cache.v_exp), 0, starts, table, lengths).float()
    bound = 1.02 * mag * (2.0 ** -10 + (max(c.lengths) + 64) * 2.0 ** -24) + 1.01 * 2.0 ** -8 * plain.float().abs()
    assert bool(((out.float() - plain.float()).abs() <= 2 * bound).all())
    assert bool(((lse - plse).abs() <= 2 * (2.0 ** -11 + (max(c.lengths) + 64) * 2.0 ** -24 + 2.0 ** -22 * (plse.abs() + 30.0))).all())


@pytest.mark.parametrize("group", [1, 8, 40])
def test_hints_choose_no_tokens(group):
    """Hints that are too small or far too large: the same tokens."""
    rng = np.random.default_rng([22, group])
    c = Groups([(1500, [(2, 300), (1, 20), (5, 40)]), (200, [(3, 700)] * 2)], 32, rng)
    pool = oc.new_pool(1, c.pages, 1, 128, 32)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, group, 128), "f16")
    cache, starts, table, lengths = to_gpu(pool), ids(c.starts), ids(c.table), ids(c.lengths)
    shared = mdss.cache_shared(cache, c.T, starts, table, lengths, ids(c.groups))
    want = oc.attention(pool, 0, q64, c.starts, c.table, c.lengths, 128 ** -0.5)
    for most in ((1, 1, 1, 1), (5, 1, 64, 100000), (1, 1000, 100000, 1), (1000000, 64, 1, 64), (1, 64, 640, 0)):
        out, lse = mdss.cache_attention_shared(q, cache, 0, starts, table, lengths, shared, want_lse=True,
                                               **dict(zip(("max_new", "max_group", "max_shared", "max_own"), most)))
        check(out, lse, want, "f16", 128, max(c.lengths))


def test_strides_scales_and_a_workspace():
    rng = np.random.default_rng(18)
    c = Groups([(200, [(2, 9), (1, 30)]), (90, [(1, 2)] * 3)], 16, rng)
    pool = oc.new_pool(1, c.pages, 2, 64, 16)
    fill(pool, rng)
    wide, wide64 = queries(rng, (c.T, 8, 64), "bf16")
    run(pool, c, wide[:, 2:6], wide64[:, 2:6], "bf16", scale=0.3)
    out = torch.empty((c.T, 4, 64), dtype=torch.bfloat16, device="cuda:0")
    space = torch.empty(1 << 22, dtype=torch.uint8, device="cuda:0")
    got = run(pool, c, wide[:, 4:], wide64[:, 4:], "bf16", scale=-0.2, out=out, workspace=space)
    assert got.data_ptr() == out.data_ptr()
    odd = torch.zeros(wide.numel() + 3, dtype=torch.bfloat16, device="cuda:0")
    odd[3:] = wide.reshape(-1)
    run(pool, c, odd[3:].view(c.T, 8, 64), wide64, "bf16")


def test_a_plan_serves_later_steps():
    """Rows grow by a token a step while their leading pages stay: what was found at the first step holds."""
    rng = np.random.default_rng(19)
    c = Groups([(300, [(1, 20), (1, 30), (1, 5)])], 16, rng, extra=2)
    pool = oc.new_pool(1, c.pages, 1, 64, 16)
    fill(pool, rng)
    cache = to_gpu(pool)
    shared = mdss.cache_shared(cache, 3, None, ids(c.table), ids(c.lengths), ids(c.groups))
    for step in range(3):
        q, q64 = queries(rng, (3, 4, 64), "bf16")
        out, lse = mdss.cache_attention_shared(q, cache, 0, None, ids(c.table), ids(c.lengths), shared, want_lse=True)
        check(out, lse, oc.attention(pool, 0, q64, c.starts, c.table, c.lengths, 0.125), "bf16", 64, 400)
        c.lengths = [x + 1 for x in c.lengths]


def test_another_stream_and_a_graph():
    rng = np.random.default_rng(20)
    c = Groups([(3000, [(1, 100), (1, 700)]), (700, [(1, 3)] * 3)], 16, rng)
    pool = oc.new_pool(1, c.pages, 2, 64, 16)
    fill(pool, rng)
    cache, table, lengths, groups = to_gpu(pool), ids(c.table), ids(c.lengths), ids(c.groups)
    q, _ = queries(rng, (c.T, 8, 64), "bf16")

    def call():
        return mdss.cache_attention_shared(q, cache, 0, None, table, lengths, mdss.cache_shared(cache, c.T, None, table, lengths, groups))

    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert torch.equal(got, want)
    graphs = []
    for _ in range(2):  # two graphs have scratch of their own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        graphs.append((graph, got))
    for _ in range(3):
        for graph, got in graphs:
            got.zero_()
        torch.cuda.synchronize()
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got, want) for _, got in graphs)
        torch.randn(1000, device="cuda:0").sum().item()
