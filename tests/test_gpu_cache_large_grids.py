"""Attention calls of more row tiles and heads than one launch holds (2^24 workgroups): within the documented sizes, so they run."""
import pytest
import torch

import paper_2410_18234_amd as mdss
from cache_cases import ids

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ragged", [False, True])
def test_many_sequences_of_many_heads(ragged):
    """56000 x 300 workgroups.  All sequences lie on one page, with the same query: rows differ by their lengths alone."""
    S, heads, d = 56000, 300, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    cache = mdss.PagedCache.empty(1, 1, heads, d, 16)
    cache.k.copy_(torch.randint(0, 0x60, cache.k.shape, generator=g, device="cuda", dtype=torch.uint8))
    cache.v.copy_(torch.randint(0, 0x60, cache.v.shape, generator=g, device="cuda", dtype=torch.uint8))
    cache.k_exp.fill_(-6)
    cache.v_exp.fill_(0)
    q = torch.randn((1, heads, d), generator=g, device="cuda").bfloat16()
    lengths = torch.randint(1, 17, (S,), generator=g, device="cuda", dtype=torch.int32)
    table = torch.zeros((S, 1), dtype=torch.int32, device="cuda")
    few = mdss.cache_attention(q.expand(16, -1, -1), cache, 0, None, table[:16], ids(range(1, 17)))
    assert len({row.tobytes() for row in few.view(torch.int16).cpu().numpy()}) == 16
    starts = torch.arange(S + 1, dtype=torch.int32, device="cuda") if ragged else None
    out = mdss.cache_attention(q.expand(S, -1, -1), cache, 0, starts, table, lengths, max_new=1)
    assert torch.equal(out, few[lengths.long() - 1])
