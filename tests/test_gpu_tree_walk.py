"""psa_tree_attention where one CTA's share of the work is hundreds of short row tiles, among them many without keys, beside trees with NaN among their values: what a CTA's roles tell each other
about one item must not reach the next one or the one before.  Against attention over the held values in 64 bits; tolerances as in test_gpu_tree.py."""
import random

import pytest
import torch

import drafts_reference as ref
import serving_reference as sref
from paper_2012_01114_b200 import binding as psa
from test_gpu_cache import Made, _queries

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
G, D, PAGE = 64, 32, 16
HELD = [100, 128, 40, 128, 17]                   # of the sequences with trees, the last ones with a NaN in a value of the tree's token 1


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("empty", ["no keys", "no slot"])
@pytest.mark.parametrize("run", [1, 3, 40])
def test_many_short_items_in_one_share(run, empty):
    """`run` sequences without keys ahead of each with a tree.  A row tile without keys counts 11 units of work, one with 128 keys as much; the last sequence, of which nothing is asked but its length,
    makes a CTA's share (its units over the number of CTAs) larger than all others together."""
    r = random.Random(run)
    c = Made(HELD, 1, D, PAGE, 31, extra_slots=3)
    spare = [s for s in range(len(HELD) + 3) if s not in c.slot]
    sizes = [r.choice([2, 3, 12, 17]) if n < 100 else r.choice([2, 64, 100]) for n in HELD]
    trees = [[i - 1 for i in range(n)] if b % 2 else ref.random_tree(n, r)[0] for b, n in enumerate(sizes)]
    for b in (3, 4):
        lens = c.lens.clone()
        lens[c.slot[b]] = HELD[b] - sizes[b] + 2
        V = torch.randn(1, 1, D, device="cuda").to(BF)
        V[0, 0, 7] = float("nan")
        psa.psa_cache_append(torch.randn(1, 1, D, device="cuda").to(BF), V, c.pool, c.tables, lens, _ints([c.slot[b]]), sref.starts([1]), PAGE)
    seqs, parents, counts, of = [], [], [], []
    while len(seqs) < 320:
        for b, tree in enumerate(trees):
            for _ in range(run):
                n = r.choice([1, 2, 5])
                seqs.append(spare[0] if empty == "no keys" else r.choice([-1, 99]))
                parents += [-1] * n
                counts.append(n)
                of.append(None)
            seqs.append(c.slot[b])
            parents += tree
            counts.append(len(tree))
            of.append(b)
    seqs, parents, counts, of = seqs[:400], parents, counts[:400], of[:400]
    parents = parents[:sum(counts)]
    units = sum(-(-n * G // 128) * 11 for n in counts)
    tiles = 160 * units // (32 * 2) + 1          # of the last sequence, 64 rows a token of 64: 32 row tiles, each 2 units or more a tile of keys
    seqs, parents, counts = seqs + [spare[1]], parents + [i - 1 for i in range(64)], counts + [64]
    tables = torch.full((len(HELD) + 3, tiles * 128 // PAGE), -1, dtype=torch.int32, device="cuda")
    tables[:, :c.tables.shape[1]] = c.tables
    tables[spare[1]] = c.tables[c.slot[1], 0]    # (one page over and over)
    lens = c.lens.clone()
    lens[spare[0]], lens[spare[1]] = 0, tiles * 128
    Q, starts, seqs, parents = _queries(sum(counts), G, D, BF, 3), sref.starts(counts), _ints(seqs), _ints(parents)
    first = None
    for _ in range(20):
        lse = torch.full((sum(counts), G), float("nan"), device="cuda")
        out = psa.psa_tree_attention(Q, c.pool, tables, lens, seqs, starts, parents, 1, PAGE, 100, lse=lse)
        assert psa.psa_last_issued()[0] == (psa.OK if empty == "no keys" else psa.ERR_SHAPE)
        if first is not None:
            assert torch.equal(out.view(torch.int16), first[0].view(torch.int16)) and torch.equal(lse, first[1])
        first = out, lse
    wanted, at = {}, 0
    for n, b in zip(counts, of):
        o, l = out[at:at + n], lse[at:at + n]
        if b is None:
            assert (o == 0).all() and (l == -torch.inf).all()
        else:
            seen = ref.seen_by(trees[b], n, HELD[b])
            if b >= 3:                           # the rows that see the NaN: their group of channels, that is all of d = 32
                bad = seen[:, HELD[b] - n + 1]
                assert bad.any() and torch.isnan(o[bad.cuda()]).all()
                keep = ~bad
            else:
                keep = torch.ones(n, dtype=torch.bool)
            at0 = at
            q = Q[at0:at0 + n]
            key = (b, at0)
            if len([k for k in wanted if k[0] == b]) < 4 or not keep.any():      # (the 64-bit form of a few of them; of the others that nothing is missing)
                wanted[key] = True
                if keep.any():
                    k, v = c.k[b].clone(), c.v[b].clone()
                    if b >= 3:                   # (rows that do not see the token that was written again: whatever it holds)
                        v[HELD[b] - n + 1] = 0
                    sref.close(o[keep.cuda()], None, [x[keep] for x in ref.attend(q, k, v, D ** -0.5, seen)], BF, HELD[b], 2 * 2.0 ** -11 + 2.0 ** -8)
            assert torch.isfinite(o[keep.cuda()]).all() and torch.isfinite(l).all()
        at += n
