"""psa_verify_drafts against its definition in 64 bits: whole numbers, equal wherever no decision is nearer to its border than 1e-9 (sums of 64-bit exponentials: each 2^-52, in another order)."""
import random

import numpy as np
import pytest
import torch

import drafts_reference as ref
import serving_reference as sref
from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Made:
    def __init__(self, sizes, V, dtype=torch.float32, seed=0, branch=3, depth=6, spread=2.0, stride=0, distinct=True):
        r, g = random.Random(seed), torch.Generator().manual_seed(seed)
        self.sizes, self.V, rows = sizes, V, sum(sizes)
        self.trees = [ref.random_tree(n, r, depth, branch)[0] for n in sizes]
        buf = [torch.zeros(rows, V + stride, dtype=dtype) for _ in range(2)]
        self.logits, self.drafts = (x[:, stride // 2:stride // 2 + V] for x in buf)
        self.logits.copy_((spread * torch.randn(rows, V, generator=g)).to(dtype))
        self.drafts.copy_((self.logits.float() + 0.7 * torch.randn(rows, V, generator=g)).to(dtype))
        self.uniform = torch.rand(rows, generator=g)
        self.tokens, at = [], 0
        for tree in self.trees:
            for i, p in enumerate(tree):
                if i == 0:
                    self.tokens.append(r.randrange(V))
                    continue
                before = [self.tokens[at + k] for k in range(i) if tree[k] == p and k > 0]
                q = torch.softmax(self.drafts[at + max(p, 0)].double(), 0)
                if distinct and len(before) < V:
                    q[before] = 0
                self.tokens.append(int(torch.multinomial(q, 1, generator=g)))
            at += len(tree)
        self.cuda = {k: x.cuda()[:, stride // 2:stride // 2 + V] for k, x in zip(("logits", "drafts"), buf)}

    def run(self, drafts, temperatures, distinct=True, tokens=None, parents=None, **kw):
        return psa.psa_verify_drafts(self.cuda["logits"], _ints(self.tokens if tokens is None else tokens), _ints([p for t in self.trees for p in t] if parents is None else parents),
                                     sref.starts(self.sizes), self.uniform.cuda(), drafts=self.cuda["drafts"] if drafts else None,
                                     temperatures=None if temperatures is None else torch.tensor(temperatures, dtype=torch.float32, device="cuda"), distinct=distinct, **kw)

    def check(self, drafts, temperatures=None, distinct=True, status=psa.OK):
        path, accepted, following = (x.tolist() for x in self.run(drafts, temperatures, distinct))
        assert psa.psa_last_issued()[0] == status
        at, sure, stood = 0, 0, 0
        for b, (n, tree) in enumerate(zip(self.sizes, self.trees)):
            if n == 0:
                assert (accepted[b], following[b]) == (0, -1)
                continue
            T = 1.0 if temperatures is None else float(torch.tensor(temperatures[b], dtype=torch.float32))
            p, k, x, margin = ref.verify(self.logits[at:at + n], self.drafts[at:at + n] if drafts else None, self.tokens[at:at + n], tree, self.uniform[at:at + n], T, distinct)
            if margin > 1e-9:
                assert (path[at:at + n], accepted[b], following[b]) == (p + [-1] * (n - len(p)), k, x), (b, margin)
                sure += 1
                stood += k
            at += n
        return sure, stood


@pytest.mark.parametrize("kind", ["certain", "distinct", "replaced"])
@pytest.mark.parametrize("V,dtype", [(1, "f32"), (2, "bf16"), (7, "f16"), (33, "f32"), (1000, "bf16"), (2049, "f16"), (8193, "f32"), (50001, "bf16")])
def test_trees(V, dtype, kind):
    sizes = [1, 2, 0, 9, 30, 5, 12, 1, 17, 3] * (1 if V > 5000 else 5)
    m = Made(sizes, V, TYPES[dtype], V, distinct=kind != "replaced")
    r = random.Random(V)
    sure, stood = m.check(kind != "certain", [r.choice([0.0, 0.5, 0.8, 1.0, 1.7]) for _ in sizes], kind == "distinct")
    assert sure >= 0.8 * sum(n > 0 for n in sizes)
    assert stood > 0 or kind == "certain" or V < 5000                # (a drawn token of tens of thousands is no likely one: as a certain draft it hardly ever stands)


@pytest.mark.parametrize("V,seqs", [(150001, 2), (128000, 40), (260000, 100), (5000, 300)])
def test_sizes(V, seqs):
    """Vocabularies shared by clusters of all sizes, and parts too long to be kept."""
    rows = 3 if V > 20000 else 6
    m = Made([rows if b % 2 else 1 for b in range(seqs)] if V * seqs > 1e7 else [rows] * seqs, V, torch.float32, V, spread=3.0)
    assert m.check(True)[0] >= 0.9 * seqs


@pytest.mark.parametrize("temperature", [1e-3, 0.01, 0.03])
@pytest.mark.parametrize("kind", ["certain", "distinct", "replaced"])
def test_siblings_behind_a_likely_one(kind, temperature):
    """Drafts of which one token is nearly certain, and siblings drawn from the 1e-6 to 1e-40 that it leaves; the large model likes all tokens alike, or as the drafts do."""
    for spread in (0.0, 2.0):
        m = Made([20, 9, 33, 5] * 4, 96, torch.bfloat16, 31, branch=8, depth=3, spread=spread, distinct=kind != "replaced")
        assert m.check(kind != "certain", [temperature] * 16, kind == "distinct")[0] > 0


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("stride", [0, 1, 2, 3, 5, 6, 14])
def test_strides_and_alignment(stride, dtype):
    m = Made([7, 4, 12], 4099, TYPES[dtype], stride, stride=stride)
    m.check(True)
    m.check(False, [0.0, 1.0, 0.7])


def test_likeliest_token_of_equal_ones_is_the_first():
    m = Made([4] * 6, 9000, torch.bfloat16, 1, spread=0.3)          # (bf16 and a narrow spread: many equal numbers)
    top = m.logits.float().amax(-1)
    assert ((m.logits.float() == top[:, None]).sum(-1) > 1).any()
    assert m.check(False, [0.0] * 6)[0] == 6


@pytest.mark.parametrize("kind", ["certain", "distinct", "replaced"])
def test_masked_tokens(kind):
    """-inf for most tokens, for all but one, and for drafted ones."""
    m = Made([6] * 8, 5000, torch.float32, 3)
    for b, keep in enumerate((1, 2, 3, 50, 1, 5, 400, 4999)):
        rows = slice(6 * b, 6 * b + 6)
        mask = torch.ones(5000, dtype=torch.bool)
        mask[torch.randperm(5000, generator=torch.Generator().manual_seed(b))[:keep]] = False
        m.logits[rows, mask] = -torch.inf
        if b % 2:
            m.drafts[rows, mask] = -torch.inf
    m.cuda = dict(logits=m.logits.cuda(), drafts=m.drafts.cuda())
    assert m.check(kind != "certain", None, kind == "distinct")[0] >= 6


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), None])
@pytest.mark.parametrize("where", ["logits", "drafts"])
@pytest.mark.parametrize("temperature", [0.0, 1.0])
def test_rows_that_are_no_distribution(where, bad, temperature):
    """On the path: it ends there.  Off the path, and drafts behind a leaf: not looked at."""
    m = Made([5, 5, 5], 3000, torch.float32, 4)
    m.trees = [[-1, 0, 1, 2, 3], [-1, 0, 0, 0, 0], [-1, 0, 1, 2, 3]]
    rows = getattr(m, where)
    for row in (0, 9):                           # the first sequence's root, and a leaf of the second
        if bad is None:
            rows[row] = -torch.inf
        else:
            rows[row, 1234] = bad
    m.uniform[5:10] = 0.99999                    # (nobody stands there)
    m.tokens[5:10] = [0, *m.logits[5].argsort()[:4].tolist()]
    m.cuda = dict(logits=m.logits.cuda(), drafts=m.drafts.cuda())
    reads = where == "logits" or temperature > 0
    m.check(True, [temperature] * 3, status=psa.ERR_NUMERIC if reads else psa.OK)
    path, accepted, following = m.run(True, [temperature] * 3)
    assert (accepted[0] == 0 and following[0] == -1 and path[:5].tolist() == [0, -1, -1, -1, -1]) if reads else following[0] >= 0
    assert following[1] >= 0 and following[2] >= 0


def test_arguments_that_are_reported():
    m = Made([4, 4, 4, 4], 500, torch.float32, 5)
    tokens = list(m.tokens)
    tokens[5] = 500
    tokens[6] = -1
    _, accepted, following = m.run(True, None, tokens=tokens)
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE and (following >= 0).all()
    parents = [p for t in m.trees for p in t]
    parents[9], parents[11] = 3, -4              # (of itself, and below -1: not reached)
    _, accepted, following = m.run(True, None, parents=parents)
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE and (following >= 0).all()
    for T in (-1.0, float("nan"), float("inf")):
        path, accepted, following = m.run(True, [1.0, T, 1.0, 0.0])
        assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
        assert (following[1], accepted[1], path[4:8].tolist()) == (-1, 0, [-1] * 4) and (following[[0, 2, 3]] >= 0).all()


def test_trees_that_are_too_large():
    m = Made([1024, 3], 64, torch.float32, 6, branch=2, depth=30)
    m.check(True)
    m = Made([1025, 3], 64, torch.float32, 6, branch=2, depth=30)
    path, accepted, following = m.run(True, None)
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE and following[0] == -1 and accepted[0] == 0 and (path[:1025] == -1).all() and following[1] >= 0


def test_rows_behind_the_last_sequence_and_no_rows():
    m = Made([3, 2], 100, torch.float32, 7)
    path = torch.full((5,), 77, dtype=torch.int32, device="cuda")
    psa.psa_verify_drafts(m.cuda["logits"], _ints(m.tokens), _ints([p for t in m.trees for p in t]), _ints([0, 3]), m.uniform.cuda(), path)
    assert (path[3:] == 77).all() and (path[:3] != 77).all()
    empty = torch.empty(0, 100, device="cuda")
    _, accepted, following = psa.psa_verify_drafts(empty, _ints([]), _ints([]), _ints([0, 0, 0]), torch.empty(0, device="cuda"))
    assert accepted.tolist() == [0, 0] and following.tolist() == [-1, -1]


def test_more_sequences_than_a_grid_has_rows():
    n, V = 66000, 40
    g = torch.Generator(device="cuda").manual_seed(8)
    logits, u = torch.randn(n, V, device="cuda", generator=g), torch.rand(n, device="cuda", generator=g)
    _, accepted, following = psa.psa_verify_drafts(logits, torch.zeros(n, dtype=torch.int32, device="cuda"), torch.full((n,), -1, dtype=torch.int32, device="cuda"),
                                                   torch.arange(n + 1, dtype=torch.int32, device="cuda"), u)
    sums = torch.softmax(logits.double(), -1).cumsum(-1)
    sums = sums / sums[:, -1:]
    near = (sums - u.double()[:, None]).abs().amin(-1) < 1e-12
    assert (accepted == 0).all() and (torch.where(near, following.long(), (sums > u.double()[:, None]).int().argmax(-1)) == following).all() and near.sum() < 5


@pytest.mark.parametrize("kind", ["certain", "distinct", "replaced"])
def test_the_targets_distribution(kind):
    """200,000 sequences of a root with two children of it and a grandchild: the first token behind the root has the target's probabilities, whatever was drafted.  Five standard deviations
    of each count."""
    n, V = 200000, 6
    g = torch.Generator(device="cuda").manual_seed(9)
    row, draft = torch.randn(V, device="cuda", generator=g), torch.randn(V, device="cuda", generator=g)
    logits, drafts = row.repeat(4 * n, 1), draft.repeat(4 * n, 1)
    q = torch.softmax(draft.double(), -1)
    tokens = torch.zeros(n, 4, dtype=torch.int32, device="cuda")
    tokens[:, 1:3] = torch.multinomial(q.repeat(n, 1), 2, replacement=kind == "replaced", generator=g).int()
    parents = _ints([-1, 0, 0, 1]).repeat(n)
    u = torch.rand(4 * n, device="cuda", generator=g)
    path, accepted, following = psa.psa_verify_drafts(logits, tokens.view(-1), parents, torch.arange(0, 4 * n + 1, 4, dtype=torch.int32, device="cuda"), u,
                                                      drafts=None if kind == "certain" else drafts, distinct=kind == "distinct")
    second = path.view(n, 4)[:, 1].long()
    first = torch.where(accepted > 0, tokens.gather(1, second.clamp(min=0)[:, None])[:, 0], following)
    count, p = torch.bincount(first.long(), minlength=V).double().cpu() / n, torch.softmax(row.double(), -1).cpu()
    assert (count - p).abs().le(5 * (p * (1 - p) / n).sqrt()).all() and 0.05 < (accepted > 0).double().mean() < 0.999


def test_captured_and_on_another_stream():
    m = Made([9, 4, 20], 30000, torch.bfloat16, 10)
    want = [x.clone() for x in m.run(True, [1.0, 0.0, 0.8])]
    args = (m.cuda["logits"], _ints(m.tokens), _ints([p for t in m.trees for p in t]), sref.starts(m.sizes), m.uniform.cuda())
    T = torch.tensor([1.0, 0.0, 0.8], device="cuda")
    out = [torch.zeros_like(x) for x in want]
    call = lambda: psa.psa_verify_drafts(*args, *out, drafts=m.cuda["drafts"], temperatures=T)  # noqa: E731
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        call()
    for _ in range(2):
        for x in out:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
