"""The pages of a cache against the same bookkeeping done one sequence at a time on the host (tests/serving_reference.py): whole numbers, equal."""
import random

import pytest
import torch

import serving_reference as ref
from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu


class Both:
    def __init__(self, slots, width, pages, page_size, layers=2, page_bytes=160, seed=0):
        pool = torch.randint(0, 256, (layers, pages, page_bytes), dtype=torch.uint8, generator=torch.Generator().manual_seed(seed))
        self.book = ref.Book(slots, width, pages, page_size, pool.clone())
        self.tables, self.lens = torch.full((slots, width), -1, dtype=torch.int32, device="cuda"), torch.zeros(slots, dtype=torch.int32, device="cuda")
        self.refs, self.pool, self.short = torch.zeros(pages, dtype=torch.int32, device="cuda"), pool.cuda(), torch.full((1,), -5, dtype=torch.int32, device="cuda")
        self.size = page_size

    def _list(self, x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def free(self, seqs):
        self.book.free(seqs)
        psa.psa_pages_free(self.tables, self.lens, self.refs, self._list(seqs), self.size)

    def fork(self, parents, children):
        self.book.fork(parents, children)
        psa.psa_pages_fork(self.tables, self.lens, self.refs, self._list(parents), self._list(children), self.size)

    def reserve(self, seqs, add):
        want = self.book.reserve(seqs, add)
        psa.psa_pages_reserve(self.tables, self.lens, self.refs, self.pool, self._list(seqs), self._list(add), self.size, self.short)
        assert int(self.short) == want
        return want

    def compact(self, in_place=True):
        want, live = self.book.compact(), torch.full((1,), -1, dtype=torch.int32, device="cuda")
        t, r, p = (self.tables, self.refs, self.pool) if in_place else (torch.empty_like(self.tables), torch.empty_like(self.refs), torch.empty_like(self.pool))
        old = [x.clone() for x in (self.tables, self.refs, self.pool)]
        psa.psa_pages_compact(self.tables, self.refs, self.pool, t, r, p, live)
        assert int(live) == want
        if not in_place:
            assert all(torch.equal(a, b) for a, b in zip(old, (self.tables, self.refs, self.pool)))
            p[:, want:] = self.pool[:, want:]
            self.tables, self.refs, self.pool = t, r, p
        return want

    def same(self, pool=True):
        assert psa.psa_last_issued()[0] == psa.OK
        assert self.tables.tolist() == self.book.t and self.lens.tolist() == self.book.l and self.refs.tolist() == self.book.r
        if pool:
            assert torch.equal(self.pool.cpu(), self.book.pool)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("seed", range(4))
def test_a_server_at_random(seed, in_place):
    r = random.Random(seed)
    b = Both(40, 9, 120, r.choice([16, 32]), seed=seed)
    alive = []
    for step in range(60):
        what = r.random()
        if what < 0.45:
            new = [s for s in range(40) if s not in alive][:r.randint(0, 3)]
            seqs = r.sample(alive, min(len(alive), r.randint(0, 12))) + new
            room = [9 * b.size - b.book.l[s] for s in seqs]
            if seqs and b.reserve(seqs, [min(x, r.choice([0, 1, 1, 5, 16, 40])) for x in room]) == 0:
                alive += new
        elif what < 0.65 and alive:
            children = [s for s in range(40) if s not in alive][:r.randint(1, 6)]
            if children:
                b.fork([r.choice(alive) for _ in children], children)
                alive += children
        elif what < 0.85 and alive:
            gone = r.sample(alive, r.randint(1, len(alive) // 2 + 1))
            b.free(gone)
            alive = [s for s in alive if s not in gone]
        else:
            n = b.compact(in_place)
            assert all(x > 0 for x in b.book.r[:n]) and not any(b.book.r[n:])
            # the pool's places behind the live pages hold whatever they held
            b.book.pool[:, n:] = b.pool.cpu()[:, n:]
        b.same()


def test_branches_of_one_sequence():
    """Ten children of one parent with a partly filled page, all extended in one call with the parent: ten copies, and one that keeps the page."""
    b = Both(11, 4, 40, 16)
    b.reserve([0], [21])
    b.fork([0] * 10, list(range(1, 11)))
    b.same()
    b.reserve(list(range(11)), [1] * 11)
    b.same()
    assert len(set(b.tables[:, 1].tolist())) == 11 and len(set(b.tables[:, 0].tolist())) == 1


def test_nothing_changes_when_pages_are_missing():
    b = Both(4, 8, 5, 16)
    assert b.reserve([0, 1], [40, 16]) == 0
    assert b.reserve([2, 0, 1], [30, 30, 0]) == 3          # two pages each for the first two, one is left
    b.same()
    assert b.reserve([0, 2], [8, 16]) == 0
    b.same()


def test_page_edges_and_empty_lists():
    b = Both(3, 4, 12, 16)
    for add in (16, 0, 15, 1, 1, 31):
        b.reserve([1], [add])
        b.same()
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    psa.psa_pages_free(b.tables, b.lens, b.refs, empty, 16)
    psa.psa_pages_fork(b.tables, b.lens, b.refs, empty, empty, 16)
    psa.psa_pages_reserve(b.tables, b.lens, b.refs, b.pool, empty, empty, 16, b.short)
    psa.psa_pages_copy(b.pool, b.pool, empty, empty)
    b.free([0, 1, 2])
    b.same()
    assert b.compact() == 0
    b.same(pool=False)


def test_many_sequences_and_a_large_pool():
    b = Both(3000, 3, 70000, 16, layers=1, page_bytes=16)
    b.refs[:66000] = 1                     # (held by somebody else)
    b.book.r[:66000] = [1] * 66000
    r = random.Random(3)
    assert b.reserve(list(range(0, 3000, 2)), [r.randint(0, 40) for _ in range(1500)]) == 0
    b.fork(list(range(0, 3000, 4)), list(range(1, 3000, 4)))
    b.reserve(list(range(3000)), [r.randint(0, 3) for _ in range(3000)])
    b.same()
    b.refs[:66000:2] = 0
    b.book.r[:66000:2] = [0] * 33000
    b.compact()
    b.same(pool=False)


@pytest.mark.parametrize("page_bytes,layers", [(16, 1), (160, 3), (20480, 2), (163840, 1), (40000, 2)])
def test_copy(page_bytes, layers):
    g = torch.Generator(device="cuda").manual_seed(1)
    a, c = (torch.randint(0, 256, (layers, n, page_bytes), dtype=torch.uint8, device="cuda", generator=g) for n in (9, 14))
    src, dst = torch.tensor([3, 3, 0, 8], dtype=torch.int32, device="cuda"), torch.tensor([13, 1, 2, 0], dtype=torch.int32, device="cuda")
    want = c.clone()
    want[:, dst.long()] = a[:, src.long()]
    psa.psa_pages_copy(a, c, src, dst)
    assert psa.psa_last_issued()[0] == psa.OK and torch.equal(c, want)
    want[:, 5] = want[:, 13]
    psa.psa_pages_copy(c, c, dst[:1], dst[:1] * 0 + 5)
    assert torch.equal(c, want)


def test_arguments_that_name_nothing():
    b = Both(4, 4, 12, 16)
    b.reserve([0, 1], [20, 5])
    one = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for bad in (-1, 4, 1 << 30):
        for call in (lambda: psa.psa_pages_free(b.tables, b.lens, b.refs, one(bad), 16), lambda: psa.psa_pages_fork(b.tables, b.lens, b.refs, one(bad), one(2), 16),
                     lambda: psa.psa_pages_fork(b.tables, b.lens, b.refs, one(0), one(bad), 16),
                     lambda: psa.psa_pages_reserve(b.tables, b.lens, b.refs, b.pool, one(0, bad), one(1, 1), 16, b.short),
                     lambda: psa.psa_pages_copy(b.pool, b.pool, one(bad if bad != 4 else 12), one(2))):
            call()
            assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
    psa.psa_pages_fork(b.tables, b.lens, b.refs, one(0), one(1), 16)          # slot 1 holds pages
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
    psa.psa_pages_reserve(b.tables, b.lens, b.refs, b.pool, one(0), one(60), 16, b.short)      # beyond the table
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
    psa.psa_pages_free(b.tables, b.lens, b.refs, one(2), 16)
    b.same()
    b.tables[2, 0] = 12                                                       # a page that the pool does not have
    psa.psa_pages_free(b.tables, b.lens, b.refs, one(2), 16)
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
    psa.psa_pages_free(b.tables, b.lens, b.refs, one(2), 16)
    b.same()


def test_graph_replay():
    b = Both(6, 6, 40, 16)
    b.reserve([0, 1], [20, 33])
    parents, children, add = b._list([0, 1, 1]), b._list([2, 3, 4]), b._list([3, 1, 20])
    psa.psa_pages_free(b.tables, b.lens, b.refs, children, 16)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        psa.psa_pages_free(b.tables, b.lens, b.refs, children, 16)
        psa.psa_pages_fork(b.tables, b.lens, b.refs, parents, children, 16)
        psa.psa_pages_reserve(b.tables, b.lens, b.refs, b.pool, children, add, 16, b.short)
    for _ in range(3):
        graph.replay()
        b.book.free([2, 3, 4])
        b.book.fork([0, 1, 1], [2, 3, 4])
        assert b.book.reserve([2, 3, 4], [3, 1, 20]) == int(b.short) == 0
        b.same()


@pytest.mark.parametrize("n", [255, 256, 257, 700])
def test_long_lists_that_share_pages(n):
    """Children of three parents with a partly filled page each, in the order of chance: with the parents in the list the last one keeps the page, without one parent all copy."""
    b = Both(n + 3, 3, 2 * n + 20, 16, layers=1, page_bytes=16)
    b.reserve([0, 1, 2], [21, 5, 16])
    b.fork([i % 3 for i in range(n)], [3 + i for i in range(n)])
    r = random.Random(n)
    every = list(range(1, n + 3))
    r.shuffle(every)
    for _ in range(2):
        assert b.reserve(every[:n], [1 if r.random() < 0.9 else 0 for _ in range(n)]) == 0
        b.same()
