"""The drafting operators together, as examples/drafts.py uses them: every pass against the same attention over the held values in 64 bits, so that a pass sees what the ones before it have left in
the cache.  Of the 2-norm: 2^-8 / sqrt(3) for the output's rounding to bf16, and as much again for the weights' in the prompt pass or for the held values', which are compared as bf16:
3.2e-3; 4e-3 are allowed."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "drafts.py")


def _example():
    spec = importlib.util.spec_from_file_location("drafts_example", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


@pytest.mark.parametrize("prompts,tokens,temperature", [(3, 24, 0.8), (1, 10, 0.0), (6, 30, 1.5)])
def test_answers(prompts, tokens, temperature):
    errors, answers = _example().main(prompts, tokens, temperature, say=lambda *a: None)
    assert max(errors) <= 4e-3, errors
    assert all(len(a) >= tokens and min(a) >= 0 for a in answers)
    assert len(errors) - 1 < max(len(a) for a in answers) - 1            # (drafts stand now and then)


def test_the_likeliest_tokens_are_those_without_drafts():
    """At temperature 0 a pass gives the tokens that one at a time gives: logits are formed in fp32 from attention in bf16, whose roundings differ by 2^-8 of one of two terms.  The answer's own tokens
    are looked at one after another, and compared with the likeliest ones wherever the two likeliest do not lie nearer to each other than 2^-6 of the largest logit."""
    example = _example()
    _, answers = example.main(2, 12, 0.0, say=lambda *a: None)
    g = torch.Generator(device="cuda").manual_seed(1)
    lengths = [int(n) for n in torch.randint(1, 200, (2,), generator=torch.Generator().manual_seed(2))]
    model, slots = example.Model(2), example._ints([0, 1])
    given = torch.randint(0, example.VOCAB, (sum(lengths),), dtype=torch.int32, device="cuda", generator=g)
    logits, _ = model.look(given, slots, lengths)
    rows, compared = logits[torch.tensor(lengths, device="cuda").cumsum(0) - 1], 0
    for i in range(12):
        top = rows.topk(2, -1)
        for b in range(2):
            if top.values[b, 0] - top.values[b, 1] > 2.0 ** -6 * rows[b].abs().max():
                assert answers[b][i] == int(top.indices[b, 0])
                compared += 1
        rows, _ = model.look(example._ints([a[i] for a in answers]), slots, [1, 1], example._ints([-1, -1]), example._ints([0, 0]))
    assert compared >= 6
