"""Lengths that the program takes back (guessed tokens that were refused) and sequences that grow again: no page is lost, none is written to that another sequence shares."""
import random

import pytest
import torch

import serving_reference as ref
import test_gpu_pages as pages
from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu


class Book(ref.Book):
    """Pages behind a length are given back when the sequence is in a list."""

    def reserve(self, seqs, add):
        for s in seqs:
            for c in range(-(-self.l[s] // self.size), len(self.t[s])):
                if self.t[s][c] < 0:
                    break
                self.r[self.t[s][c]] -= 1
                self.t[s][c] = -1
        return super().reserve(seqs, add)


class Both(pages.Both):
    def __init__(self, *a, **kw):
        super().__init__(*a, **kw)
        self.book = Book(self.tables.shape[0], self.tables.shape[1], self.refs.numel(), self.size, self.book.pool)

    def take_back(self, s, n):
        self.lens[s] -= n
        self.book.l[s] -= n

    def whole(self):
        """Every reference is a table's."""
        count = torch.zeros_like(self.refs).cpu()
        for p in self.tables[self.tables >= 0].tolist():
            count[p] += 1
        assert torch.equal(count, self.refs.cpu())


def test_one_sequence():
    b = Both(2, 8, 9, 16)
    for add, back in ((20, 5), (40, 30), (1, 26), (100, 100), (128, 17), (17, 128), (0, 0)):
        assert b.reserve([0], [add]) == 0
        b.take_back(0, back)
        b.same()
        b.whole()
    assert b.reserve([0, 1], [33, 96]) == 0                  # (all nine pages)
    b.same()
    b.whole()


def test_own_pages_are_enough_in_a_full_pool():
    b = Both(2, 8, 4, 16)
    assert b.reserve([0, 1], [48, 16]) == 0
    b.take_back(0, 32)
    assert b.reserve([0], [49]) == 2                         # (two given back, four asked for)
    b.same()
    b.whole()
    assert b.reserve([0], [32]) == 0
    b.same()
    b.whole()


@pytest.mark.parametrize("n", [3, 300])
def test_shared_pages_behind_a_length(n):
    """A fork made after tokens were taken back shares the pages behind the length as well: both sequences grow, each into a page of its own."""
    b = Both(2 * n, 5, 12 * n, 16)
    own, children = list(range(n)), list(range(n, 2 * n))
    assert b.reserve(own, [40] * n) == 0
    for s in own:
        b.take_back(s, 20 + s % 5)                           # a partly filled page and one behind it, or 16 tokens and two
    b.fork(own, children)
    b.same()
    b.whole()
    assert b.reserve(children, [30] * n) == 0
    b.same()
    b.whole()
    assert b.reserve(own + children, [3] * n + [5] * n) == 0
    b.same()
    b.whole()
    b.free(own)
    b.compact()
    b.same(pool=False)
    b.whole()


@pytest.mark.parametrize("seed", range(4))
def test_drafts_at_random(seed):
    r = random.Random(seed)
    b = Both(30, 9, 100, r.choice([16, 32]), seed=seed)
    b.reserve([0], [0])                                      # (a call, for whose status `same` asks)
    alive = []
    for step in range(60):
        what = r.random()
        if what < 0.5:
            new = [s for s in range(30) if s not in alive][:r.randint(0, 3)]
            seqs = r.sample(alive, min(len(alive), r.randint(0, 12))) + new
            if seqs and b.reserve(seqs, [min(9 * b.size - b.book.l[s], r.choice([0, 1, 1, 5, 16, 40])) for s in seqs]) == 0:
                alive += new
        elif what < 0.7:
            for s in r.sample(alive, len(alive) // 2):
                b.take_back(s, min(b.book.l[s], r.choice([1, 4, 16, 50])))
        elif what < 0.8 and alive:
            children = [s for s in range(30) if s not in alive][:r.randint(1, 6)]
            if children:
                b.fork([r.choice(alive) for _ in children], children)
                alive += children
        elif what < 0.9 and alive:
            gone = r.sample(alive, r.randint(1, len(alive) // 2 + 1))
            b.free(gone)
            alive = [s for s in alive if s not in gone]
        else:
            n = b.compact()
            b.book.pool[:, n:] = b.pool.cpu()[:, n:]
        b.same()
        b.whole()


def test_nothing_is_given_back_by_a_list_with_a_bad_entry():
    b = Both(3, 4, 12, 16)
    b.reserve([0, 1], [48, 48])
    b.take_back(0, 40)
    one = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for seqs, add in (((0, 7), (30, 1)), ((0, 1), (30, 40))):
        psa.psa_pages_reserve(b.tables, b.lens, b.refs, b.pool, one(*seqs), one(*add), 16, b.short)
        assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
    b.tables[0, 2] = 12                                      # behind the length, a page that the pool does not have
    psa.psa_pages_reserve(b.tables, b.lens, b.refs, b.pool, one(0), one(30), 16, b.short)
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
    b.tables[0, 2] = b.book.t[0][2]
    assert b.reserve([1], [0]) == 0
    b.same()
