"""The example of a speculative step on the paged cache: the drafted run gives the tokens of the plain one, its pages come back."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_drafting_changes_the_steps_and_not_the_tokens():
    import speculative_cache as example
    prompt = list(range(3, 60))
    one, steps, _, pages = example.generate(prompt, 24, 0)
    got, fewer, taken, pages_too = example.generate(prompt, 24, 3)
    assert len(one) == len(got) == 24 and steps == 23 and fewer <= steps
    assert all(0 <= t < example.VOCAB for t in one + got)
    assert taken == 0 or fewer < steps
    assert got == one
    held = -(-(len(prompt) + 24) // example.PAGE)
    assert pages in (held - 1, held) and pages_too in (held - 1, held, held + 1)
