"""The loops of test_gpu_shared_decode.py without the hint max_shared, which sends calls as small as those to the attention that knows no
prefixes: forked rows go over what they share together, by the kernels of prefixes and the join (`near`'s bound holds for them: a
prefix of up to seven tiles by at most four waves, or one where it has more than 64 rows, and own tokens by at most four)."""
import pytest

import paper_2410_18234_amd as mdss
import test_gpu_shared_decode as loops
from test_gpu_beam_decode import example  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture
def calls(monkeypatch):
    """The calls' hints, max_shared left out."""
    real, seen = mdss.cache_attention_shared, []

    def without(*args, max_shared, **kw):
        assert max_shared > 0
        seen.append(args)
        return real(*args, **kw)

    monkeypatch.setattr(mdss, "cache_attention_shared", without)
    return seen


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("ps,d,drafts,tokens", [(16, 64, 4, 3), (32, 128, 2, 6), (64, 128, 12, 2)])
def test_drafts_of_a_step(ps, d, drafts, tokens, interleaved, calls):
    loops.test_drafts_of_a_step(ps, d, drafts, tokens, interleaved)
    assert len(calls) == 4 and all(max(shared[0].tolist()) >= 256 for *_, shared in calls)


@pytest.mark.parametrize("ps,beams", [(16, 4), (32, 3)])
def test_beams_share_their_prompts(example, ps, beams, calls):  # noqa: F811
    loops.test_beams_share_their_prompts(example, ps, beams)
    assert len(calls) == 40 and all(max(shared[0].tolist()) >= 128 for *_, shared in calls)
