"""psa_tree_attention against attention over the held values in 64 bits.  Rounded on the way to an output: the weight and the held value to fp16 (2^-11 each), the result to its type
(tests/serving_reference.py)."""
import random

import pytest
import torch

import drafts_reference as ref
import serving_reference as sref
from paper_2012_01114_b200 import binding as psa
from test_gpu_cache import Made, _queries

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(params=["sixteens", "tiles"], autouse=True)
def form(request, monkeypatch):
    """Both kernels: which one runs goes by the most rows and by the keys that the tables have room for."""
    monkeypatch.setitem(FORM, "tiles", request.param == "tiles")


FORM = {}


def _made(*args):
    c = Made(*args)
    if FORM["tiles"]:
        c.tables = torch.nn.functional.pad(c.tables, (0, 32768 // c.page - c.tables.shape[1]), value=-1)
    return c


def _most(n):
    return 1024 if FORM["tiles"] else n


def _trees(sizes, seed=0, **kw):
    r = random.Random(seed)
    return [ref.random_tree(n, r, **kw)[0] for n in sizes]


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _attend(c, trees, G, dtype, Q=None, max_q=None, scale=None, lse=None, out=None, parents=None):
    n = [len(t) for t in trees]
    Q = _queries(sum(n), c.Hkv * G, c.d, dtype, 3) if Q is None else Q
    parents = _ints([p for t in trees for p in t]) if parents is None else parents
    return Q, psa.psa_tree_attention(Q, c.pool, c.tables, c.lens, c.seqs, sref.starts(n), parents, c.Hkv, c.page, _most(max(n + [1])) if max_q is None else max_q, scale=scale, out=out, lse=lse)


def _check(c, trees, G, dtype, Q=None, max_q=None, scale=None, status=psa.OK):
    n = [len(t) for t in trees]
    lse = torch.full((sum(n), c.Hkv * G), float("nan"), device="cuda")
    Q, out = _attend(c, trees, G, dtype, Q, max_q, scale, lse)
    assert psa.psa_last_issued()[0] == status
    at = 0
    for tree, k, v in zip(trees, c.k, c.v):
        if tree:
            r = ref.attend(Q[at:at + len(tree)], k, v, c.d ** -0.5 if scale is None else scale, ref.seen_by(tree, len(tree), len(k)))
            sref.close(out[at:at + len(tree)], lse[at:at + len(tree)], r, dtype, len(k), 2 * 2.0 ** -11 + sref.UNIT[dtype])
        at += len(tree)
    return out


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("G,Hkv,d,page", [(1, 2, 32, 16), (1, 1, 64, 64), (4, 2, 128, 16), (8, 1, 128, 64), (3, 3, 96, 48), (8, 2, 256, 32), (9, 1, 64, 16), (20, 1, 128, 32), (64, 1, 64, 128), (5, 2, 32, 32)])
def test_trees(G, Hkv, d, page, dtype):
    """Also trees of one token, none, as many as are held, and more than are held (the first ones have no place, and their descendants see what there is)."""
    lens, sizes = [1, 15, 33, 64, 200, 0, 333, 6, 130], [1, 7, 33, 20, 13, 3, 0, 9, 64]
    _check(_made(lens, Hkv, d, page, d), _trees(sizes, d), G, dtype)


@pytest.mark.parametrize("d,G", [(64, 4), (128, 8), (128, 1), (96, 2), (256, 2)])
def test_long_and_short_together(d, G):
    """Rows that are cut into parts, the tree at the end of the last one, beside short ones; the same twice."""
    lens, sizes = [6000, 40, 900, 1], [26, 5, 64, 1]
    c = _made(lens, 2, d, 64, 7)
    a = _check(c, _trees(sizes, 1), G, BF)
    assert torch.equal(a, _check(c, _trees(sizes, 1), G, BF))


@pytest.mark.parametrize("G,d", [(1, 128), (4, 64), (4, 128)])
def test_where_the_tree_begins(G, d):
    """Every offset of the tree's first token inside a step of 32 tokens and a tile of 128, and trees that fill words of 32 bits."""
    lens = list(range(40, 73)) + [127, 128, 129, 160, 255, 256, 257]
    c = _made(lens, 1, d, 16, 9)
    for size in (1, 2, 31, 32, 33):
        _check(c, _trees([size] * len(lens), size), G, HF)


def test_shapes_of_trees():
    c = _made([70, 90, 64, 80], 2, 64, 16, 11)
    n = 40
    chain, star, forest = [i - 1 for i in range(n)], [-1] + [0] * (n - 1), [-1] * n
    _check(c, [chain, star, forest, _trees([n], 5, forest=True)[0]], 4, BF)


def test_a_chain_is_the_causal_form():
    c = _made([50, 300, 17], 2, 128, 16, 12)
    n = [5, 3, 4]
    Q, out = _attend(c, [[i - 1 for i in range(k)] for k in n], 2, BF)
    want = c.attend(Q, n, max_q=5)
    assert ((out.double() - want.double()).abs() <= 2.0 ** -6 * want.double().abs() + 2.0 ** -10).all()


def test_large_trees():
    c = _made([1500, 1024, 1030], 1, 64, 64, 13)
    r = random.Random(2)
    trees = [[i - 1 for i in range(1024)], ref.random_tree(1000, r, depth=40)[0], ref.random_tree(517, r)[0]]
    _check(c, trees, 2, BF)


def test_one_that_is_too_large_is_left_out():
    c = _made([1500, 40, 60], 1, 64, 64, 14)
    trees = [[i - 1 for i in range(1025)], _trees([7])[0], _trees([9], 1)[0]]
    n = [len(t) for t in trees]
    out = torch.full((sum(n) + 3, 2 * 64), 9.0, dtype=BF, device="cuda")
    Q = _queries(sum(n) + 3, 2, 64, BF)
    parents = _ints([p for t in trees for p in t] + [0] * 3)
    psa.psa_tree_attention(Q, c.pool, c.tables, c.lens, c.seqs, sref.starts(n), parents, 1, 64, _most(9), out=out)
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
    assert (out[:1025] == 9).all() and (out[-3:] == 9).all()
    assert torch.isfinite(out[1025:-3]).all() and not (out[1025:-3] == 9).any(-1).any()


def test_parents_that_are_none():
    """Later tokens, itself and numbers below -1: taken for -1, and reported."""
    c = _made([60], 1, 64, 16, 15)
    bad = [-1, 0, 2, -7, 3, 9, 5, 1 << 30]
    good = [-1, 0, -1, -1, 3, -1, 5, -1]
    Q, out = _attend(c, [good], 4, BF)
    _, got = _attend(c, [bad], 4, BF, Q)
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
    assert torch.equal(out, got)


@pytest.mark.parametrize("G,n", [(1, 6), (4, 6), (4, 40)])
@pytest.mark.parametrize("which", [0, 1])
def test_a_nan_is_seen_by_its_descendants(which, G, n):
    c = _made([100], 1, 64, 16, 16)
    tree = ref.random_tree(n, random.Random(4))[0]
    K, V = torch.randn(1, 1, 64, device="cuda").to(BF), torch.randn(1, 1, 64, device="cuda").to(BF)
    Q, plain = _attend(c, [tree], G, BF)
    bad = 2                                      # the tree's token 2
    lens = c.lens.clone()
    lens[c.slot[0]] = 100 - n + bad + 1
    (K, V)[which][0, 0, 40] = float("nan")
    psa.psa_cache_append(K, V, c.pool, c.tables, lens, c.seqs, sref.starts([1]), 16)
    _, out = _attend(c, [tree], G, BF, Q)
    seen = ref.seen_by(tree, n, 100)[:, 100 - n + bad].cuda()
    assert torch.equal(out[~seen], plain[~seen]) and seen.any()
    got = torch.isnan(out[seen].view(-1, G, 64))
    assert got.all() if which == 0 else (got[..., 32:].all() and not got[..., :32].any())


def test_scale_strides_and_small_numbers():
    c = _made([50, 700], 2, 64, 16, 17)
    trees = _trees([9, 30], 6)
    _check(c, trees, 4, BF, scale=0.9)
    _check(_made([2500, 5000], 1, 64, 16, 23), trees, 4, BF, scale=0.9)
    buf = _queries(39, 20, 64, BF, 5)
    _check(c, trees, 4, BF, Q=buf[:, 4:12])
    for size in (1e-30, 1e-6, 1e6):
        _check(c, trees, 4, BF, Q=(_queries(39, 8, 64, BF, 6) * size).to(BF), scale=0.125 / size)


@pytest.mark.parametrize("G", [1, 4])
def test_bounds_that_are_too_small_or_large(G):
    c = _made([50, 700, 90], 2, 128, 16, 18)
    trees = _trees([9, 30, 2], 7)
    for max_q in (1, 30, 1024):
        _check(c, trees, G, BF, max_q=max_q)


def test_many_sequences():
    r = random.Random(19)
    lens = [r.choice([0, 3, 40, 130, 300]) for _ in range(600)]
    _check(_made(lens, 1, 32, 16, 19), _trees([r.choice([0, 1, 5, 12, 40]) for _ in lens], 8), 2, BF)


def test_missing_pages_and_slots():
    """Tokens of a page that does not exist are left out; a slot that does not exist has no tokens; both are reported."""
    c = _made([60, 50, 40], 1, 64, 16, 20)
    trees = _trees([6, 4, 5], 9)
    Q, good = _attend(c, trees, 4, BF)
    c.tables[c.slot[0], 1] = -1
    c.tables[c.slot[1], 0] = 1 << 20
    c.seqs[2] = -3
    _, out = _attend(c, trees, 4, BF, Q)
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
    for b, (at, n, gone) in enumerate(((0, 6, range(16, 32)), (6, 4, range(0, 16)))):
        seen = ref.seen_by(trees[b], n, len(c.k[b]))
        seen[:, list(gone)] = False
        sref.close(out[at:at + n], None, ref.attend(Q[at:at + n], c.k[b], c.v[b], 0.125, seen), BF, 60, 2 * 2.0 ** -11 + 2.0 ** -8)
    assert (out[10:] == 0).all() and torch.isfinite(good).all()


def test_captured_and_on_another_stream():
    c = _made([2000, 90], 2, 128, 64, 21)
    trees = _trees([20, 9], 10)
    parents = _ints([p for t in trees for p in t])
    Q, want = _attend(c, trees, 4, BF, parents=parents)
    out, s = torch.zeros_like(want), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    starts = sref.starts([20, 9])
    call = lambda: psa.psa_tree_attention(Q, c.pool, c.tables, c.lens, c.seqs, starts, parents, 2, 64, _most(20), out=out)  # noqa: E731
    with torch.cuda.stream(s):
        call()
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        call()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert psa.psa_last_issued()[0] == psa.OK


def test_starts_that_descend_are_reported():
    c = _made([60, 50], 1, 64, 16, 22)
    Q = _queries(10, 4, 64, BF)
    out = torch.full((10, 256), 3.0, dtype=BF, device="cuda")
    psa.psa_tree_attention(Q, c.pool, c.tables, c.lens, c.seqs, _ints([0, 8, 5]), _ints([-1] * 10), 1, 16, _most(8), out=out)
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE and (out == 3).all()
