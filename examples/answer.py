"""Answers with one attention layer: the serving operators as a program uses them, on random weights.

    python examples/answer.py [--prompts 3] [--tokens 8] [--branches 2]

A batch of prompts of different lengths goes through the layer in one packed pass; its keys and values go into a paged cache of 4 bits.  Then every sequence is
answered token by token, branches off halfway (the branches share pages until they write to them), and the sequences that end give their pages back.
Printed is how far each step lies from the same step over the numbers that the cache holds, in 64 bits.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2012_01114_b200 import binding as psa  # noqa: E402

HEADS, KV_HEADS, D, PAGE = 8, 2, 64, 16


class Layer:
    """Projections of one attention layer and the cache of its keys and values."""

    def __init__(self, slots, pages, width, d_model=256, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.w = (torch.randn(d_model, (HEADS + 2 * KV_HEADS) * D, device="cuda", generator=g) * d_model ** -0.5).bfloat16()
        self.d_model = d_model
        self.tables = torch.full((slots, width), -1, dtype=torch.int32, device="cuda")
        self.lens, self.refs = torch.zeros(slots, dtype=torch.int32, device="cuda"), torch.zeros(pages, dtype=torch.int32, device="cuda")
        self.pool = torch.zeros(pages, psa.psa_cache_page_bytes(KV_HEADS, PAGE, D), dtype=torch.uint8, device="cuda")
        self.short = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.held = {}                           # for the comparison: what the cache holds, by slot

    def step(self, x, seqs, counts, prompt):
        """x [tokens, d_model], packed: counts[i] tokens for slot seqs[i] -> attention output [tokens, HEADS * D].  prompt: the slots hold nothing yet."""
        slots, starts = _ints(seqs), _ints([0] + torch.tensor(counts).cumsum(0).tolist())
        rows = (x @ self.w).view(-1, HEADS + 2 * KV_HEADS, D)
        q, k, v = rows[:, :HEADS], rows[:, HEADS:HEADS + KV_HEADS], rows[:, HEADS + KV_HEADS:]
        k_held, v_held = torch.empty_like(k.contiguous()), torch.empty_like(v.contiguous())
        psa.psa_pages_reserve(self.tables, self.lens, self.refs, self.pool, slots, _ints(counts), PAGE, self.short)
        psa.psa_cache_append(k, v, self.pool, self.tables, self.lens, slots, starts, PAGE, k_held=k_held, v_held=v_held)
        if prompt:                               # the prompt attends to what the cache will hold, as the steps after it do
            out = psa.psa_prompt_attention(q, k_held, v_held, starts)
        else:
            out = psa.psa_cache_attention(q, self.pool, self.tables, self.lens, slots, starts, KV_HEADS, PAGE, max_q=max(counts))
        return out, self._error(q, k_held, v_held, out, seqs, counts)

    def fork(self, parents, children):
        psa.psa_pages_fork(self.tables, self.lens, self.refs, _ints(parents), _ints(children), PAGE)
        self.held.update({c: self.held[p] for p, c in zip(parents, children)})

    def free(self, seqs):
        psa.psa_pages_free(self.tables, self.lens, self.refs, _ints(seqs), PAGE)

    def compact(self):
        live = torch.zeros(1, dtype=torch.int32, device="cuda")
        psa.psa_pages_compact(self.tables, self.refs, self.pool, self.tables, self.refs, self.pool, live)
        return int(live)

    def _error(self, q, k, v, out, seqs, counts):
        worst, at = 0.0, 0
        for s, n in zip(seqs, counts):
            ks, vs = (torch.cat([old, new[at:at + n].double()]) for old, new in zip(self.held.get(s, (k[:0].double(), v[:0].double())), (k, v)))
            self.held[s] = ks, vs
            kk, vv = (t.repeat_interleave(HEADS // KV_HEADS, 1) for t in (ks, vs))
            w = torch.einsum("qhd,khd->hqk", q[at:at + n].double(), kk) * D ** -0.5
            seen = torch.arange(len(ks), device="cuda") <= torch.arange(len(ks) - n, len(ks), device="cuda")[:, None]
            want = torch.einsum("hqk,khd->qhd", w.masked_fill(~seen, -torch.inf).softmax(-1), vv).reshape(n, -1)
            worst = max(worst, float((out[at:at + n].double() - want).norm() / want.norm()))
            at += n
        return worst


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def main(prompts=3, tokens=8, branches=2, say=print):
    g = torch.Generator(device="cuda").manual_seed(1)
    lengths = [int(n) for n in torch.randint(1, 200, (prompts,), generator=torch.Generator().manual_seed(2))]
    layer = Layer(slots=prompts * (1 + branches), pages=prompts * (1 + branches) * 16, width=16)
    draw = lambda n: torch.randn(n, layer.d_model, device="cuda", generator=g).bfloat16()  # noqa: E731
    alive, errors = list(range(prompts)), []
    _, e = layer.step(draw(sum(lengths)), alive, lengths, prompt=True)
    errors.append(e)
    say("prompts of %s tokens: relative difference %.2e" % (lengths, e))
    for t in range(tokens):
        if t == tokens // 2 and branches:
            parents = [s for s in range(prompts) for _ in range(branches)]
            children = list(range(prompts, prompts * (1 + branches)))
            layer.fork(parents, children)
            alive += children
            say("token %d: %d branches" % (t, len(children)))
        guesses = 1 if t % 3 else 2              # now and then two tokens at once
        _, e = layer.step(draw(guesses * len(alive)), alive, [guesses] * len(alive), prompt=False)
        errors.append(e)
        say("token %d: %d sequences, relative difference %.2e" % (t, len(alive), e))
    used = int((layer.refs > 0).sum())
    stay = alive[1::2] or alive
    layer.free([s for s in alive if s not in stay])
    left = layer.compact()
    status, _ = psa.psa_last_issued()
    _, e = layer.step(draw(len(stay)), stay, [1] * len(stay), prompt=False)
    errors.append(e)
    say("%d pages in use, %d after every other sequence has ended and the rest has moved together: relative difference %.2e" % (used, left, e))
    assert status == psa.OK and int(layer.short) == 0
    return errors


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("prompts", 3), ("tokens", 8), ("branches", 2)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    main(a.prompts, a.tokens, a.branches)
