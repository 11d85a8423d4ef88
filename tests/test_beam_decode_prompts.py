"""examples/beam_decode.py refuses prompts without a token (the logits of another prompt's last token would stand in)."""
import importlib.util
import os

import pytest

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "beam_decode.py")


@pytest.mark.parametrize("prompts", [[], [[]], [[1, 2], [], [3]]])
def test_empty_prompts(prompts):
    spec = importlib.util.spec_from_file_location("beam_decode", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    with pytest.raises(ValueError):
        module.decode(None, None, prompts, 2, 4)
