"""Attention over shared prefixes by every cut of the work: hints that are wrong, waves of rows of their own behind prefixes of few and many rows,
and the second pass of the kernel of many rows.  The bounds are those of test_gpu_cache_attention.py.

`together` repeats the rule of which calls go over what they share at all, `own_waves` that of which sequences take a wave each, for prefixes
and tables of the sizes here: a test of a kernel first shows that the call reaches it."""
import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
import test_gpu_cache_attention_shared as plain
from cache_cases import ids, to_gpu
from oracle import cache as oc
from shared_cases import Groups
from test_gpu_cache_attention import check, fill, queries

pytestmark = pytest.mark.gpu


def tiles_of(hint, tokens):
    return -(-min(hint or tokens, tokens) // 64)


def together(c, heads, group, max_group=0, max_shared=0, **_):
    rows = min(max_group or c.T, c.T) * group
    return max_shared == 0 or max_shared >= 64 and len(c.new) * heads * tiles_of(max_shared, c.table.shape[1] * c.ps) >= (49152 if rows > 64 else 12288)


def own_waves(c, heads, group, n, max_own=0, **_):
    """Few rows (up to 16 of a sequence)."""
    assert n * group <= 16
    return 1 if len(c.new) * heads >= 1024 or tiles_of(max_own, c.table.shape[1] * c.ps) <= 2 else 4


def attend(c, pool, q, heads, group, uniform=False, cache=None, **most):
    assert together(c, heads, group, **most)
    cache = to_gpu(pool) if cache is None else cache
    starts, table, lengths = None if uniform else ids(c.starts), ids(c.table), ids(c.lengths)
    shared = mdss.cache_shared(cache, c.T, starts, table, lengths, ids(c.groups))
    assert max(shared[0].tolist()) > 0
    out, lse = mdss.cache_attention_shared(q, cache, 0, starts, table, lengths, shared, want_lse=True, **most)
    torch.cuda.synchronize()
    return out, lse


def widened(c, columns):
    """Columns of no pages: a call without hints is cut for as many tokens."""
    c.table = np.pad(c.table, ((0, 0), (0, columns - c.table.shape[1])), constant_values=-1)
    return c


@pytest.mark.parametrize("d,group", [(64, 1), (128, 8), (128, 40), (256, 3)])
@pytest.mark.parametrize("most", [(1, 1, 0, 1), (5, 1, 0, 100000), (1, 1000, 0, 1), (1000000, 64, 0, 64), (0, 1, 9000, 1), (1, 1, 100000, 0), (0, 0, 100000, 64),
                                  (2, 1, 26000, 30)])
def test_hints_choose_no_tokens(most, d, group):
    """Hints that are too small or far too large, in calls that go over what they share together."""
    most = dict(zip(("max_new", "max_group", "max_shared", "max_own"), most))
    rng = np.random.default_rng([1, d, group])
    # (96 sequences of a head: 9000 tokens are 13536 of their tiles, the table's 32768 are 49152)
    c = Groups([(9500, [(2, 300), (1, 20), (5, 40)]), (200, [(3, 700)] * 2)] + [(64, [(1, 1 + i) for i in range(13)]) for _ in range(7)], 32, rng)
    widened(c, 1024)
    pool = oc.new_pool(1, c.pages, 1, d, 32)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, group, d), "f16")
    out, lse = attend(c, pool, q, 1, group, **most)
    check(out, lse, oc.attention(pool, 0, q64, c.starts, c.table, c.lengths, d ** -0.5), "f16", d, max(c.lengths))


@pytest.mark.parametrize("d,group,W", [(64, 2, 130), (128, 2, 130), (128, 8, 130), (96, 4, 130), (256, 1, 130), (64, 2, 5), (128, 4, 5), (256, 2, 5)])
def test_a_wave_for_each_sequence(d, group, W):
    """1040 (sequence, head) pairs behind one prefix of many rows, or 26 of few; tails of one to five tiles."""
    rng = np.random.default_rng([2, d, group, W])
    heads = 8
    c = Groups([(640 + 64 * (g % 3), [(1, 1 + int(x)) for x in rng.integers(0, 300, W)]) for g in range(130 // W)], 64, rng)
    assert own_waves(c, heads, group, 1) == 1
    pool = oc.new_pool(1, c.pages, heads, d, 64)
    fill(pool, rng)
    q, q64 = queries(rng, (c.T, heads * group, d), "bf16")
    out, lse = attend(c, pool, q, heads, group, uniform=True)
    check(out, lse, oc.attention(pool, 0, q64, c.starts, c.table, c.lengths, d ** -0.5), "bf16", d, max(c.lengths))


WAVES = dict(max_own=1)  # (an understatement where tails are longer: a wave takes them whole)
CASES = [(plain.test_bytes_past_the_tokens_are_never_seen, ()), (plain.test_missing_pages, ()), (plain.test_nan_reaches_only_the_rows_that_see_it, (2,)),
         (plain.test_nan_reaches_only_the_rows_that_see_it, (40,)), (plain.test_queries_that_are_not_finite, (2,)), (plain.test_queries_that_are_not_finite, (40,)),
         (plain.test_pages_of_unlike_scale_and_large_scores, ("bf16",)), (plain.test_pages_of_unlike_scale_and_large_scores, ("f16",)),
         (plain.test_long_prefix_and_long_tails, ("bf16",)), (plain.test_strides_scales_and_a_workspace, ())]
CASES += [(plain.test_prefix_lengths, (n,)) for n in (63, 64, 65, 191, 1000)]
CASES += [(plain.test_ragged_groups, (*x, "f16")) for x in ((64, 16, 2, 1), (96, 32, 2, 3), (128, 64, 8, 2), (256, 32, 1, 2))]
CASES += [(plain.test_rows_of_every_kernel, (*x, d)) for d in (64, 96, 128, 256) for x in ((2, 1, 1), (17, 1, 2), (7, 3, 4), (65, 1, 8))]


@pytest.mark.parametrize("most", [{}, WAVES], ids=["true", "waves"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join([c[0].__name__[5:], *map(str, c[1])]))
def test_together(case, most, monkeypatch):
    """The cases of test_gpu_cache_attention_shared.py with their hints, but for max_shared, which would send them apart: short tails
    go by waves of their own, behind prefixes of few rows and of many, and with `waves` all tails of up to 32 rows."""
    real = plain.hints

    def without(c, tokens, rows):
        kept = {k: v for k, v in real(c, tokens, rows).items() if k != "max_shared"}
        return {**kept, **most}

    monkeypatch.setattr(plain, "hints", without)
    case[0](*case[1])


# ---------------------------------------------------------------- the second pass of the kernel of many rows
def few_and_many(d, wide, ps, rng, prefix, more):
    """One group of three tokens with `group` query heads: rows beyond 64, or (wide) 39 of them behind a long table, which go 16 to a
    wave.  Returns the rows, the group and the rows of a wave."""
    c = Groups([(prefix, [(1, x) for x in more])], ps, rng)
    if not wide:
        return c, 40, 16 if d > 128 else 32
    widened(c, -(-24576 * 64 // ps))
    return c, 13, 16


SECOND = [(64, False), (96, False), (128, False), (256, False), (64, True), (128, True), (256, True)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("d,wide", SECOND)
def test_pages_of_unlike_scale(d, wide, kind):
    """Values of one page hide another's in f16's range; scores that one token takes.  (Those leave out of a row what
    test_gpu_shared_decode.py's `near` says, and have its bound: a row has its prefix's wave and four of its own tokens here.)"""
    rng = np.random.default_rng([3, d, wide])
    c, group, _ = few_and_many(d, wide, 64, rng, 640, (40, 3, 100))
    pool = oc.new_pool(1, c.pages, 1, d, 64)
    q, q64 = queries(rng, (3, group, d), kind)
    for scale, k_exp, v_exp in ((d ** -0.5, None, [-40, -20, -6, 0, 8]), (0.02, 3, None), (0.06, 2, [-30, -6])):
        fill(pool, rng)
        if k_exp is not None:
            pool["k_exp"][...] = k_exp
        if v_exp is not None:
            pool["v_exp"][...] = rng.choice(v_exp, pool["v_exp"].shape)
        out, lse = attend(c, pool, q, 1, group, uniform=True, scale=scale)
        ref, rlse, mag, slack = oc.attention(pool, 0, q64, c.starts, c.table, c.lengths, scale)
        more = 0.25 * mag.max(axis=2, keepdims=True) if k_exp is not None else 0.0
        check(out, lse, (ref, rlse, mag + more, slack), kind, d, max(c.lengths))


@pytest.mark.parametrize("leading", ["all", "one wave", "a row", "every other wave"])
@pytest.mark.parametrize("lead", [17.5, 24.0, 30.0])
@pytest.mark.parametrize("d,wide", SECOND)
def test_a_leading_token_without_values(d, wide, lead, leading):
    """A token of the prefix leads by far in some of the rows, and its values are 0: what the others add up to is beneath f16's
    normal range in the waves of those rows, which go over their tokens again, and in no other's."""
    rng = np.random.default_rng([4, d, wide, int(lead * 2)])
    ps = 64
    c, group, wave = few_and_many(d, wide, ps, rng, 1280, (30, 2, 65))
    pool = oc.new_pool(1, c.pages, 1, d, ps)
    for at in (0, 777):
        L = max(c.lengths)
        for page in range(c.pages):
            codes = np.zeros((ps, d))
            codes[:, 1] = rng.uniform(-1.0, 1.0, ps)
            values = rng.uniform(0.25, 4.0, (ps, d))
            if page == c.table[0, at // ps]:
                codes[at % ps], values[at % ps] = 0.0, 0.0
                codes[at % ps, 0] = 1.0
            oc.put_tokens(pool, "k", 0, page, 0, oc.encode(codes * 2.0 ** 8))
            oc.put_tokens(pool, "v", 0, page, 0, oc.encode(values * 2.0 ** 6))
        pool["k_exp"][...], pool["v_exp"][...] = -8, -6
        rows = np.arange(3 * group)
        led = {"all": rows >= 0, "one wave": rows // wave == 1, "a row": rows == 2 * wave + 3, "every other wave": rows // wave % 2 == 0}[leading]
        q = torch.zeros((3, group, d), dtype=torch.bfloat16)
        q[..., 0] = torch.from_numpy(np.where(led, lead, 0.0)).view(3, group)
        q[..., 1] = 1.0
        out, lse = attend(c, pool, q.cuda(), 1, group, uniform=True, scale=1.0)
        check(out, lse, oc.attention(pool, 0, q.double().numpy(), c.starts, c.table, c.lengths, 1.0), "bf16", d, L)


def test_new_tokens_past_token_0():
    """Tokens before starts[0] and behind the last sequence belong to nobody, and are left as they are."""
    rng = np.random.default_rng(5)
    c = Groups([(300, [(3, 20), (2, 70), (0, 4)]), (700, [(4, 9)] * 3)], 16, rng)
    pool = oc.new_pool(1, c.pages, 2, 64, 16)
    fill(pool, rng)
    T = c.T + 60
    for group in (2, 20):
        q, q64 = queries(rng, (T, 2 * group, 64), "bf16")
        cache, starts, table, lengths = to_gpu(pool), c.starts + 37, ids(c.table), ids(c.lengths)
        shared = mdss.cache_shared(cache, T, ids(starts), table, lengths, ids(c.groups))
        assert min(shared[0].tolist()) == 256
        out = torch.full((T, 2 * group, 64), 5.0, dtype=torch.bfloat16, device="cuda:0")
        _, lse = mdss.cache_attention_shared(q, cache, 0, ids(starts), table, lengths, shared, want_lse=True, out=out)
        torch.cuda.synchronize()
        mine = slice(37, 37 + c.T)
        check(out[mine], lse[mine], oc.attention(pool, 0, q64[mine], c.starts, c.table, c.lengths, 0.125), "bf16", 64, max(c.lengths))
        assert bool((out[:37] == 5.0).all()) and bool((out[37 + c.T:] == 5.0).all())
