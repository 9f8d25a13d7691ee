"""Answers with drafted tokens: one attention layer on random weights, its cache in 4 bits, and a cheap model that drafts trees of tokens for it.

    python examples/drafts.py [--prompts 3] [--tokens 24] [--temperature 0.8]

Prompts of different lengths go through the layer, their keys turned to their positions on the way into the cache.  Then, step by step, the cheap model drafts a tree of
tokens for every sequence (from its own probabilities, siblings without replacement), the layer looks at all of them in one pass, given random numbers decide which of them stand, and the
cache keeps those.  Printed is how many tokens a pass gave, and how far each pass lies from the same pass over the numbers that the cache holds, in 64 bits.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2012_01114_b200 import binding as psa  # noqa: E402

HEADS, KV_HEADS, D, PAGE, VOCAB, D_MODEL, WIDTH = 8, 2, 64, 16, 500, 256, 32
BRANCHES, LEVELS = 3, 2                          # of a drafted tree: children of a token, levels below the root


class Model:
    """Embedding, one attention layer with position rotation, logits; the cheap model leaves the layer out."""

    def __init__(self, slots, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
        self.tokens = normal(VOCAB, D_MODEL).bfloat16()
        self.qkv = (normal(D_MODEL, (HEADS + 2 * KV_HEADS) * D) * D_MODEL ** -0.5).bfloat16()
        self.out = (normal(HEADS * D, D_MODEL) * (HEADS * D) ** -0.5).bfloat16()
        self.step = (normal(D_MODEL, D_MODEL) * D_MODEL ** -0.5).bfloat16()
        self.freqs = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
        self.tables = torch.full((slots, WIDTH), -1, dtype=torch.int32, device="cuda")
        self.lens, self.refs = torch.zeros(slots, dtype=torch.int32, device="cuda"), torch.zeros(slots * WIDTH, dtype=torch.int32, device="cuda")
        self.pool = torch.zeros(slots * WIDTH, psa.psa_cache_page_bytes(KV_HEADS, PAGE, D), dtype=torch.uint8, device="cuda")
        self.short = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.held = {}                           # for the comparison: what the cache holds, by slot

    def _logits(self, x, attended=None):
        y = x.float() @ self.step.float()
        if attended is not None:
            y = y + attended.float() @ self.out.float()
        return y @ self.tokens.float().T * (2 * D_MODEL ** -0.5 / VOCAB ** 0.25)

    def draft(self, tokens):
        return self._logits(self.tokens[tokens.long()])

    def look(self, tokens, slots, sizes, parents=None, depths=None):
        """One pass over `sizes` new tokens of each slot: logits [tokens, VOCAB], and the attention's distance from the 64-bit form.  parents None: prompts, the slots hold nothing yet."""
        x, starts, counts = self.tokens[tokens.long()], _starts(sizes), _ints(sizes)
        rows = (x @ self.qkv).view(-1, HEADS + 2 * KV_HEADS, D)
        q, k, v = rows[:, :HEADS], rows[:, HEADS:HEADS + KV_HEADS], rows[:, HEADS + KV_HEADS:]
        k_held, v_held = torch.empty_like(k.contiguous()), torch.empty_like(v.contiguous())
        psa.psa_pages_reserve(self.tables, self.lens, self.refs, self.pool, slots, counts, PAGE, self.short)
        q = psa.psa_cache_append_rotary(k, v, self.pool, self.tables, self.lens, slots, starts, PAGE, self.freqs, Q=q, depths=depths, k_held=k_held, v_held=v_held)
        if parents is None:
            attended = psa.psa_prompt_attention(q, k_held, v_held, starts)
        else:
            attended = psa.psa_tree_attention(q, self.pool, self.tables, self.lens, slots, starts, parents, KV_HEADS, PAGE, max_q=max(sizes))
        return self._logits(x, attended), self._error(q, k_held, v_held, attended, slots.tolist(), sizes, None if parents is None else parents.tolist())

    def _error(self, q, k, v, out, slots, sizes, parents):
        worst, at = 0.0, 0
        for s, n in zip(slots, sizes):
            ks, vs = (torch.cat([old, new[at:at + n].double()]) for old, new in zip(self.held.get(s, (k[:0].double(), v[:0].double())), (k, v)))
            self.held[s] = ks, vs
            up = [i - 1 for i in range(n)] if parents is None else parents[at:at + n]
            seen = torch.ones(n, len(ks), dtype=torch.bool)
            seen[:, -n:] = False
            for i in range(n):
                j = i
                while j >= 0:
                    seen[i, len(ks) - n + j] = True
                    j = up[j]
            kk, vv = (t.repeat_interleave(HEADS // KV_HEADS, 1) for t in (ks, vs))
            w = torch.einsum("qhd,khd->hqk", q[at:at + n].double(), kk) * D ** -0.5
            want = torch.einsum("hqk,khd->qhd", w.masked_fill(~seen.cuda(), -torch.inf).softmax(-1), vv).reshape(n, -1)
            worst = max(worst, float((out[at:at + n].double() - want).norm() / want.norm()))
            at += n
        return worst

    def keep(self, slots, sizes, path, accepted):
        psa.psa_cache_keep(self.pool, self.tables, self.lens, slots, _starts(sizes), path, accepted, KV_HEADS, PAGE)
        at = 0
        for s, n, m in zip(slots.tolist(), sizes, accepted.tolist()):
            stay = path[at:at + m + 1].long()
            self.held[s] = tuple(torch.cat([t[:-n], t[-n:][stay]]) for t in self.held[s])
            at += n


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(sizes):
    return _ints([0] + torch.tensor(sizes).cumsum(0).tolist())


def drafted(model, roots, temperature, g):
    """A tree below each root -> tokens, parents, depths, packed, and the logits that each token's children were drawn from."""
    tokens, parents, depths, logits, last = [roots[:, None]], [-1], [0], [], [0]
    for level in range(1, LEVELS + 1):
        x = model.draft(tokens[-1].reshape(-1))
        logits.append(x.view(len(roots), -1, VOCAB))
        if temperature > 0:
            chosen = torch.multinomial((x / temperature).softmax(-1), BRANCHES, generator=g)
        else:
            chosen = x.topk(BRANCHES, -1).indices
        tokens.append(chosen.int().view(len(roots), -1))
        first = len(parents)
        parents += [p for p in last for _ in range(BRANCHES)]
        depths += [level] * (len(last) * BRANCHES)
        last = list(range(first, len(parents)))
    logits.append(model.draft(tokens[-1].reshape(-1)).view(len(roots), -1, VOCAB))
    n = len(roots)
    return torch.cat(tokens, 1).reshape(-1).contiguous(), _ints(parents * n), _ints(depths * n), torch.cat(logits, 1).reshape(-1, VOCAB).contiguous(), [len(parents)] * n


def main(prompts=3, tokens=24, temperature=0.8, say=print):
    """-> the passes' errors, and the answers (lists of tokens)."""
    g = torch.Generator(device="cuda").manual_seed(1)
    lengths = [int(n) for n in torch.randint(1, 200, (prompts,), generator=torch.Generator().manual_seed(2))]
    model, slots = Model(prompts), _ints(list(range(prompts)))
    given = torch.randint(0, VOCAB, (sum(lengths),), dtype=torch.int32, device="cuda", generator=g)
    logits, e = model.look(given, slots, lengths)
    errors, temperatures = [e], torch.full((prompts,), float(temperature), device="cuda")
    say("prompts of %s tokens: relative difference %.2e" % (lengths, e))
    # the first token behind each prompt: a tree that is only its root
    _, _, root = psa.psa_verify_drafts(logits[torch.tensor(lengths, device="cuda").cumsum(0) - 1], torch.zeros_like(slots), torch.full_like(slots, -1), _starts([1] * prompts),
                                       torch.rand(prompts, device="cuda", generator=g), temperatures=temperatures)
    answers = [[t] for t in root.tolist()]
    while min(len(a) for a in answers) < tokens:
        tree, parents, depths, drafts, sizes = drafted(model, root, temperature, g)
        logits, e = model.look(tree, slots, sizes, parents, depths)
        path, accepted, after = psa.psa_verify_drafts(logits, tree, parents, _starts(sizes), torch.rand(len(tree), device="cuda", generator=g), drafts=drafts, temperatures=temperatures)
        model.keep(slots, sizes, path, accepted)
        for b, m in enumerate(accepted.tolist()):
            at = b * sizes[0]
            answers[b] += [int(tree[at + i]) for i in path[at + 1:at + m + 1].tolist()] + [int(after[b])]
        root = after
        errors.append(e)
        say("pass %d: %s tokens, relative difference %.2e" % (len(errors) - 1, [m + 1 for m in accepted.tolist()], e))
        assert model.lens.tolist() == [n + len(a) - 1 for n, a in zip(lengths, answers)]          # (the last token is not in the cache yet)
    status, _ = psa.psa_last_issued()
    assert status == psa.OK and int(model.short) == 0
    return errors, answers


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("prompts", 3), ("tokens", 24), ("temperature", 0.8)):
        p.add_argument("--" + name, type=type(value), default=value)
    a = p.parse_args()
    main(a.prompts, a.tokens, a.temperature)
