"""The serving operators together, as examples/answer.py uses them: every step against the same attention over the held values in 64 bits.  Of the 2-norm: 2^-8 / sqrt(3)
for the output's rounding to bf16 and, in the prompt pass, as much again for the weights': 3.2e-3; 4e-3 are allowed (held values are compared as bf16 throughout, whose
rounding in the prompt pass is exact and in the steps over the cache, which hold more than bf16 does, as large as the output's)."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer.py")


@pytest.mark.parametrize("prompts,tokens,branches", [(3, 8, 2), (1, 5, 0), (6, 12, 3)])
def test_answers(prompts, tokens, branches):
    spec = importlib.util.spec_from_file_location("answer_example", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    errors = example.main(prompts, tokens, branches, say=lambda *a: None)
    assert len(errors) == tokens + 2 and max(errors) <= 4e-3, errors
