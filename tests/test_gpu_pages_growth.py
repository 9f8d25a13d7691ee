"""psa_pages_reserve for whole prompts, against the bookkeeping on the host, and for lists that ask for more pages than 31 bits count."""
import random

import pytest
import torch

from paper_2012_01114_b200 import binding as psa
from test_gpu_pages import Both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("adds", [[80000], [40000, 1, 33000, 17], [16 * 2048], [16 * 2049, 5]])
def test_thousands_of_pages_for_a_sequence(adds):
    """More pages than are kept at hand for a call (2048), from a pool in which every third one is taken."""
    b = Both(len(adds) + 1, 5200, 9000, 16, layers=1, page_bytes=16)
    b.refs[::3] = 1
    b.book.r[::3] = [1] * 3000
    r = random.Random(5)
    assert b.reserve(list(range(len(adds))), adds) == 0
    b.same()
    b.fork([0], [len(adds)])
    assert b.reserve(list(range(len(adds) + 1)), [r.randint(0, 300) for _ in range(len(adds) + 1)]) == 0
    b.same()
    for s, add in ((0, 2000), (len(adds), 45000)):       # (short of pages or not: as the host has it)
        if b.book.l[s] + add <= 5200 * 16:
            b.reserve([s], [add])
            b.same()


def test_lists_that_ask_for_more_pages_than_31_bits_count():
    """Nothing changes, and the missing pages are reported, at most 2^31 - 1."""
    width, pages = 1 << 30, 100
    tables = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    lens, refs, short = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (3, pages, 1))
    pool = torch.zeros(pages, 16, dtype=torch.uint8, device="cuda")
    for n, want in ((2, (1 << 31) - pages), (3, (1 << 31) - 1)):
        short.fill_(-5)
        psa.psa_pages_reserve(tables, lens, refs, pool, torch.arange(n, dtype=torch.int32, device="cuda"), torch.full((n,), width, dtype=torch.int32, device="cuda"), 1, short)
        assert psa.psa_last_issued()[0] == psa.OK and int(short) == want
        assert not refs.any() and not lens.any() and int(tables.amax()) == -1 and int(tables.amin()) == -1
    for n in (2, 3):                                                     # (on either side of what is summed up in 32 bits)
        psa.psa_pages_reserve(tables, lens, refs, pool, torch.arange(n, dtype=torch.int32, device="cuda"), torch.tensor([(1 << 18) + n - 2, 20, 1][:n], dtype=torch.int32, device="cuda"), 1, short)
        assert int(short) == (1 << 18) + (20, 22)[n - 2] - pages and not refs.any()
    psa.psa_pages_reserve(tables, lens, refs, pool, torch.arange(2, dtype=torch.int32, device="cuda"), torch.full((2,), 50, dtype=torch.int32, device="cuda"), 1, short)
    assert int(short) == 0 and bool((refs == 1).all()) and tables[:2, :50].flatten().tolist() == list(range(100))


def test_more_than_256k_pages_for_a_sequence():
    """Summed up in 64 bits, and given."""
    b = Both(3, 300000, 600000, 1, layers=1, page_bytes=16)
    assert b.reserve([2, 0, 1], [7, 290000, 280000]) == 0
    b.same()
