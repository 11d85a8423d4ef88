"""examples/beam_decode.py: the cache's and the beams' calls run together."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "beam_decode.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("beam_decode", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("ps,beams", [(16, 4), (32, 3)])
def test_scores_are_those_of_the_sequences(example, ps, beams):
    """Every beam's sequence, run alone in one prompt call on an empty pool, has the log probability that the search gave it."""
    prompts = [list(range(5, 5 + n)) for n in (1, 33, 16)]
    tokens, B = 20, 3
    model = example.Decoder(vocab=333)
    pages = 3 * 3 + B * beams * (tokens // ps + 3)
    cache = mdss.PagedCache.empty(model.layers, pages, model.heads, model.head_dim, ps)
    out = example.decode(model, cache, prompts, beams, tokens)
    history, score = out["history"].cpu(), out["score"].cpu()
    assert np.all(np.diff(score.numpy(), axis=1) <= 0)
    assert len({tuple(h) for h in history.view(B * beams, tokens).tolist()}) >= beams  # beams of a group differ
    for b in range(B):
        assert len({tuple(h) for h in history[b].tolist()}) == beams
    # the pool after compaction: the rows' pages, counted, are the ids 0 .. used - 1
    table, refs, used = out["table"].cpu(), out["refs"].cpu(), int(out["used"])
    held = torch.bincount(table[table >= 0].long(), minlength=pages)
    assert torch.equal(held.int(), refs) and bool((refs[:used] > 0).all()) and bool((refs[used:] == 0).all())
    assert out["lengths"].tolist() == [len(prompts[b]) + tokens for b in range(B) for _ in range(beams)]
    for b in range(B):
        for w in range(beams):
            seq = prompts[b] + history[b, w].tolist()
            n = len(seq)
            alone = mdss.PagedCache.empty(model.layers, (n + ps - 1) // ps, model.heads, model.head_dim, ps)
            table1 = torch.arange(alone.pages, dtype=torch.int32, device="cuda")[None]
            lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
            h = model(alone, torch.tensor(seq, device="cuda"), torch.arange(n, device="cuda"), None, table1, lengths, n, n)
            logp = torch.log_softmax(model.logits(h).double(), 1)
            at = torch.arange(len(prompts[b]) - 1, n - 1, device="cuda")
            want = logp[at, torch.tensor(seq[len(prompts[b]):], device="cuda")].sum().item()
            # The two runs round apart: bf16 products (2^-9) and codes whose page's exponent differs while the page
            # fills (e4m3: half a step is 2^-4) move a logit of size about 3 by some 0.1 at most, 20 tokens add up.
            assert abs(want - score[b, w].item()) < 20 * 0.1


def test_command_runs(example, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["beam_decode.py", "--groups", "2", "--beams", "3", "--tokens", "9"])
    example.main()
    assert "pages in use" in capsys.readouterr().out
