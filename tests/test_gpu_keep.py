"""psa_cache_keep against moving every token's bytes one after another."""
import random

import pytest
import torch

import drafts_reference as ref
import serving_reference as sref
from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Made:
    def __init__(self, lens, sizes, Hkv, d, page, layers, seed=0):
        r = random.Random(seed)
        need = [-(-n // page) for n in lens]
        self.pages, slots, width = sum(need) + 2, len(lens) + 2, max(need + [1]) + 1
        order, self.slot = list(range(self.pages)), list(range(slots))
        r.shuffle(order)
        r.shuffle(self.slot)
        self.slot = self.slot[:len(lens)]
        self.tables, self.lens = torch.full((slots, width), -1, dtype=torch.int32), torch.full((slots,), 5, dtype=torch.int32)
        for s, n, m in zip(self.slot, lens, need):
            self.tables[s, :m] = torch.tensor([order.pop() for _ in range(m)], dtype=torch.int32)
            self.lens[s] = n
        self.pool = torch.randint(0, 256, (layers, self.pages, Hkv * page * d * 5 // 4), dtype=torch.uint8, generator=torch.Generator().manual_seed(seed))
        self.sizes, self.Hkv, self.d, self.page = sizes, Hkv, d, page
        self.paths = [[0] + sorted(r.sample(range(1, n), r.randrange(n))) if n else [] for n in sizes]
        self.dev = dict(pool=self.pool.cuda(), tables=self.tables.cuda(), lens=self.lens.cuda(), seqs=_ints(self.slot), starts=sref.starts(sizes))
        self.path = [x for n, p in zip(sizes, self.paths) for x in p + [-1] * (n - len(p))]

    def run(self, path=None, accepted=None, new_lens=None, pool=None):
        v = self.dev
        psa.psa_cache_keep(v["pool"] if pool is None else pool, v["tables"], v["lens"], v["seqs"], v["starts"], _ints(self.path if path is None else path),
                           _ints([len(p) - 1 for p in self.paths] if accepted is None else accepted), self.Hkv, self.page, new_lens=new_lens)

    def want(self, skip=()):
        pool, lens = self.pool.clone(), self.lens.clone()
        for b, (s, n, path) in enumerate(zip(self.slot, self.sizes, self.paths)):
            if b in skip or not n:
                continue
            base = int(lens[s]) - n
            for i, p in enumerate(path):
                for h in range(self.Hkv):
                    (pa, ta), (pb, tb) = ((int(self.tables[s, x // self.page]), x % self.page) for x in (base + p, base + i))
                    pool[:, pb, ref.byte_places(self.page, self.Hkv, self.d, h, tb)] = pool[:, pa, ref.byte_places(self.page, self.Hkv, self.d, h, ta)]
            lens[s] = base + len(path)
        return pool, lens

    def check(self, skip=(), status=psa.OK):
        pool, lens = self.want(skip)
        assert psa.psa_last_issued()[0] == status
        assert torch.equal(self.dev["lens"].cpu(), lens) and torch.equal(self.dev["pool"].cpu(), pool)


@pytest.mark.parametrize("Hkv,d,page,layers", [(1, 32, 16, 1), (2, 64, 16, 3), (3, 96, 48, 2), (2, 128, 32, 2), (1, 256, 16, 1)])
def test_moves(Hkv, d, page, layers):
    lens, sizes = [1, 40, 17, 64, 33, 9, 100], [1, 7, 0, 20, 33, 2, 13]
    m = Made(lens, sizes, Hkv, d, page, layers, d)
    m.run()
    m.check()


def test_many_tokens_and_sequences():
    m = Made([1100, 300], [1024, 250], 1, 32, 64, 1, 1)
    m.run()
    m.check()
    r = random.Random(2)
    lens = [r.randrange(1, 60) for _ in range(400)]
    m = Made(lens, [r.randrange(0, min(n, 12) + 1) for n in lens], 2, 32, 16, 2, 3)
    m.run()
    m.check()


def test_lengths_elsewhere_and_one_layer():
    m = Made([30, 20], [6, 5], 2, 64, 16, 1, 4)
    new = torch.full_like(m.dev["lens"], 99)
    m.run(new_lens=new, pool=m.dev["pool"][0])
    pool, lens = m.want()
    assert torch.equal(m.dev["pool"].cpu(), pool) and torch.equal(m.dev["lens"].cpu(), m.lens)
    assert new.cpu().tolist() == [int(lens[s]) if s in m.slot else 99 for s in range(len(lens))]


def test_what_is_reported():
    """Paths that do not ascend from 0 or leave the tree, counts that no tree has, unknown slots, trees larger than what is held: left as they are, the others done."""
    for change in ("order", "first", "beyond", "accepted", "negative", "slot", "short"):
        m = Made([40, 50, 30], [8, 9, 7], 2, 64, 16, 2, 5)
        m.paths[1] = [0, 2, 5]
        path = [*m.path[:8], 0, 2, 5, *[-1] * 6, *m.path[17:]]
        accepted = [len(p) - 1 for p in m.paths]
        if change == "order":
            path[9] = 5
        elif change == "first":
            path[8] = 1
        elif change == "beyond":
            path[10] = 9
        elif change == "accepted":
            accepted[1] = 9
        elif change == "negative":
            accepted[1] = -1
        elif change == "slot":
            m.dev["seqs"][1] = 1000
        else:
            m.lens[m.slot[1]] = 5
            m.dev["lens"] = m.lens.cuda()
        m.run(path, accepted)
        m.check(skip=(1,), status=psa.ERR_SHAPE)


def test_a_missing_page():
    m = Made([40], [30], 1, 32, 16, 1, 6)
    m.paths, m.path = [[0, 5, 25]], [0, 5, 25] + [-1] * 27
    m.dev["tables"][m.slot[0], 2] = -1           # (of token 35, the third one's: not moved)
    m.paths = [[0, 5]]
    pool, _ = m.want()
    m.run(accepted=[2])
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE and torch.equal(m.dev["pool"].cpu(), pool) and int(m.dev["lens"][m.slot[0]]) == 13


def test_captured():
    m = Made([40, 50], [8, 9], 2, 64, 16, 2, 7)
    path, accepted, new = _ints(m.path), _ints([len(p) - 1 for p in m.paths]), m.dev["lens"].clone()
    v = m.dev
    call = lambda: psa.psa_cache_keep(v["pool"], v["tables"], v["lens"], v["seqs"], v["starts"], path, accepted, 2, 16, new_lens=new)  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    pool, lens = m.want()
    for _ in range(2):
        v["pool"].copy_(m.pool)
        new.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(v["pool"].cpu(), pool) and all(int(new[s]) == int(lens[s]) for s in m.slot)
