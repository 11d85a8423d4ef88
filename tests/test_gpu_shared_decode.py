"""The position and prefix calls run together, as a decoding loop uses them: prompts appended with turned keys, rows forked into drafts
or beams, their tokens appended, what they share found, and attended over."""
import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from cache_cases import ids, starts_of, to_gpu, to_pool, values
from oracle import cache as oc
from oracle import rotary as orot
from test_gpu_beam_decode import example  # noqa: F401
from test_gpu_cache_attention import check, queries
from test_gpu_rotary import close, rope_of

pytestmark = pytest.mark.gpu


def near(out, lse, want, d, tokens):
    """The bound of test_gpu_cache_attention.py, and what both calls may leave out of a row: keys of unlike size make scores that lie
    hundreds apart, so weights fall below f16's range, and where a wave's sums reach its number of tokens n it does not go over
    them again: n weights rounded below 2^-14 are off by at most 2^-25 each, times codes of 448 at most, together 2^-25 448 n <
    2^-16 of the wave's largest sum of p |v|.  Prefixes of up to six tiles and the own tokens are at most eight waves' parts of a row, each
    of them at most the row's largest sum of p |v|: 8 2^-16 = 2^-13 of that, where `check` has 2^-11 of `mag`."""
    ref, rlse, mag, slack = want
    check(out, lse, (ref, rlse, mag + 0.25 * mag.max(axis=2, keepdims=True), slack), "bf16", d, tokens)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("ps,d,drafts,tokens", [(16, 64, 4, 3), (32, 128, 2, 6), (64, 128, 12, 2)])
def test_drafts_of_a_step(ps, d, drafts, tokens, interleaved):
    """Two rounds of drafts that branch from sequences of unlike length, over both layers; attention against the oracle's on
    the pool as it is then, queries against the formula, and the same rows without sharing."""
    rng = np.random.default_rng([ps, d, drafts, interleaved])
    H, G, S = 2, 4, 3
    freq = orot.frequencies(d, 10000.0, 8.0, 300)
    rope = rope_of(freq, interleaved, 1.1)
    length = [70, 333, 200]
    width = (max(length) + 4 * tokens) // ps + 3
    cache = to_gpu(oc.new_pool(2, S * width + S * drafts * 6 + 4, H, d, ps, rng))
    refs = torch.zeros(cache.pages, dtype=torch.int32, device="cuda:0")
    table = torch.full((S, width), -1, dtype=torch.int32, device="cuda:0")
    table, lengths, refs = mdss.cache_fork(cache, table, ids([0] * S), refs, grow=ids(length))
    k, _ = values(rng, (sum(length), H, d), "bf16", False)
    v, _ = values(rng, (sum(length), H, d), "bf16", False)
    for layer in range(2):
        mdss.cache_append_rotary(cache, layer, k, v, ids(starts_of(length)), table, lengths, rope)
    for step in range(2):
        rows = S * drafts
        parent = np.repeat(np.arange(S), drafts)
        old = (table, lengths, refs)
        new = [1 + (3 * i + step) % tokens for i in range(rows)]
        status = torch.zeros(rows, dtype=torch.int32, device="cuda:0")
        table, lengths, refs = mdss.cache_fork(cache, *old, ids(parent), None, ids(new), row_status=status)
        starts, T = ids(starts_of(new)), sum(new)
        at = np.concatenate([np.arange(L, L + n) for L, n in zip(np.repeat(length, drafts), new)])
        groups = ids(np.arange(S + 1) * drafts)
        shared = mdss.cache_shared(cache, T, starts, table, lengths, groups)
        assert shared[0].tolist() == [L // max(64, ps) * max(64, ps) for L in np.repeat(length, drafts)]
        for layer in range(2):
            k, _ = values(rng, (T, H, d), "bf16", False)
            v, _ = values(rng, (T, H, d), "bf16", False)
            q, q64 = queries(rng, (T, H * G, d), "bf16")
            turned = mdss.cache_append_rotary(cache, layer, k, v, starts, table, lengths, rope, q=q, row_status=status)
            close(turned, q64, freq, at, interleaved, 1.1, False, "bf16")
            most = dict(max_new=tokens, max_group=tokens * drafts, max_shared=max(length), max_own=ps + 64 + tokens)
            out, lse = mdss.cache_attention_shared(turned, cache, layer, starts, table, lengths, shared, want_lse=True, **most)
            torch.cuda.synchronize()
            want = oc.attention(to_pool(cache), layer, turned.double().cpu().numpy(), starts_of(new), table.cpu().numpy(),
                                lengths.tolist(), d ** -0.5)
            near(out, lse, want, d, max(length) + tokens)
            near(*mdss.cache_attention(turned, cache, layer, starts, table, lengths, want_lse=True), want, d, max(length) + tokens)
        assert not bool(status.any())
        # the first draft of each sequence is kept
        keep = ids(np.arange(S) * drafts)
        table, lengths, refs = mdss.cache_fork(cache, table, lengths, refs, keep)
        length = lengths.tolist()


@pytest.mark.parametrize("ps,beams", [(16, 4), (32, 3)])
def test_beams_share_their_prompts(example, ps, beams):  # noqa: F811
    """Every beam's sequence, run alone without sharing, has the log probability that the search gave it (the bound is that of
    test_gpu_beam_decode.py)."""
    prompts = [list(range(5, 5 + n)) for n in (1, 133, 70)]
    tokens, B = 20, 3
    model = example.Decoder(vocab=333, rotary=True)
    pages = 220 // ps + 6 + B * beams * (tokens // ps + 3)
    cache = mdss.PagedCache.empty(model.layers, pages, model.heads, model.head_dim, ps)
    out = example.decode(model, cache, prompts, beams, tokens, share=True)
    history, score = out["history"].cpu(), out["score"].cpu()
    assert np.all(np.diff(score.numpy(), axis=1) <= 0)
    for b in range(B):
        assert len({tuple(h) for h in history[b].tolist()}) == beams
        for w in range(beams):
            seq = prompts[b] + history[b, w].tolist()
            n = len(seq)
            alone = mdss.PagedCache.empty(model.layers, (n + ps - 1) // ps, model.heads, model.head_dim, ps)
            table1 = torch.arange(alone.pages, dtype=torch.int32, device="cuda")[None]
            h = model(alone, torch.tensor(seq, device="cuda"), None, None, table1, torch.tensor([n], dtype=torch.int32, device="cuda"), n, n)
            logp = torch.log_softmax(model.logits(h).double(), 1)
            at = torch.arange(len(prompts[b]) - 1, n - 1, device="cuda")
            want = logp[at, torch.tensor(seq[len(prompts[b]):], device="cuda")].sum().item()
            assert abs(want - score[b, w].item()) < 20 * 0.1


def test_command_runs(example, capsys, monkeypatch):  # noqa: F811
    monkeypatch.setattr("sys.argv", ["beam_decode.py", "--groups", "2", "--beams", "3", "--tokens", "9", "--rotary", "--share"])
    example.main()
    assert "pages in use" in capsys.readouterr().out
