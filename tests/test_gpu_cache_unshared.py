"""Sequences that share pages against the same ones on pages of their own: after any course of forks, cuts and appends, every row
reads the same codes and exponents, and attends to the same bits."""
import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from cache_cases import ids, to_gpu, to_pool
from oracle import cache as oc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("ps,d", [(16, 64), (32, 128)])
def test_rows_read_what_they_wrote(ps, d, seed):
    rng = np.random.default_rng([ps, seed])
    rows, H, width, vocab = 6, 2, 9, 50
    kv = rng.standard_normal((2, vocab, H, d)) * np.exp2(rng.integers(-4, 5, (2, vocab, 1, 1)))  # tokens of unlike size: exponents grow
    kv = torch.from_numpy(kv).bfloat16()
    cache = to_gpu(oc.new_pool(1, rows * width + 10, H, d, ps, rng))
    table, lengths = torch.full((rows, width), -1, dtype=torch.int32, device="cuda"), ids([0] * rows)
    refs = torch.zeros(cache.pages, dtype=torch.int32, device="cuda")
    own = [oc.new_pool(1, width, H, d, ps) for _ in range(rows)]  # row by row, page j in place j
    length = [0] * rows
    line = np.arange(width, dtype=np.int32)[None]
    status = torch.zeros(rows, dtype=torch.int32, device="cuda")
    for step in range(30):
        parent = rng.permutation(rows) if step == 0 else np.where(rng.random(rows) < 0.5, np.arange(rows), rng.integers(0, rows, rows))
        keep = [max(0, length[p] - int(rng.choice([0, 0, 0, 1, 5, ps]))) for p in parent]
        grow = [int(rng.integers(1, 3 * ps)) if step == 0 else int(rng.choice([0, 1, 1, 1, 4])) for _ in range(rows)]
        grow = [min(g, width * ps - k) for g, k in zip(grow, keep)]
        table, lengths, refs = mdss.cache_fork(cache, table, lengths, refs, ids(parent), ids(keep), ids(grow), row_status=status)
        starts = np.concatenate(([0], np.cumsum(grow)))
        tokens = rng.integers(0, vocab, starts[-1])
        k, v = kv[0][tokens], kv[1][tokens]
        mdss.cache_append(cache, 0, k.cuda(), v.cuda(), ids(starts), table, lengths, row_status=status)
        own = [{n: x.copy() for n, x in own[p].items()} for p in parent]
        length = [a + b for a, b in zip(keep, grow)]
        for i in range(rows):
            mine = slice(starts[i], starts[i + 1])
            assert oc.append(own[i], 0, k[mine].double().numpy(), v[mine].double().numpy(), [0, grow[i]], line, [length[i]]) == set()
    assert not bool(status.any()) and lengths.tolist() == length
    pool, where = to_pool(cache), table.cpu().numpy()
    for i in range(rows):
        for j in range((length[i] + ps - 1) // ps):
            m = min(ps, length[i] - j * ps)
            for n in ("k", "v"):
                assert (pool[n + "_exp"][0, where[i, j]] == own[i][n + "_exp"][0, j]).all()
                for h in range(H):
                    np.testing.assert_array_equal(oc.tokens_of(pool, n, 0, where[i, j], h)[:m], oc.tokens_of(own[i], n, 0, j, h)[:m])
    apart = to_gpu({n: np.concatenate([o[n] for o in own], axis=1) for n in own[0]})
    lined = ids(np.arange(rows * width).reshape(rows, width))
    q = torch.from_numpy(rng.standard_normal((2 * rows, 4 * H, d))).bfloat16().cuda()
    got = mdss.cache_attention(q, cache, 0, None, table, lengths, want_lse=True)
    want = mdss.cache_attention(q, apart, 0, None, lined, lengths, want_lse=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
