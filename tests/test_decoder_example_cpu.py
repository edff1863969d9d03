"""What examples/decoder.py refuses, before anything is computed: no GPU is needed."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("prompts", [[[]], [[1, 2], []], [[], [3], [4, 5]]])
def test_a_prompt_without_tokens_is_refused(prompts):
    """It has no row of its own whose hidden state its answer could begin with: another prompt's would be taken."""
    import decoder
    with pytest.raises(AssertionError, match="prompts"):
        decoder.answer(None, [1, 2, 3], prompts, 4)
