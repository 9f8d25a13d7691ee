"""psa_cache_keep with lengths that go to an array of their own: every listed slot gets its length, also those that are left as they are."""
import ctypes

import pytest
import torch

from paper_2012_01114_b200 import binding as psa
from paper_2012_01114_b200 import build

P = 1 << 20                                     # an address; nothing is read there


def _made(*args):
    from test_gpu_keep import Made
    return Made(*args)


@pytest.mark.gpu
@pytest.mark.parametrize("refused", [None, "path", "accepted", "count", "slot"])
def test_listed_slots_without_rows_and_refused_ones(refused):
    m = _made([30, 20, 17, 44, 9, 3], [6, 0, 5, 0, 9, 0], 2, 64, 16, 2, 4)
    path, accepted = list(m.path), [len(p) - 1 for p in m.paths]
    if refused == "path":
        path[6] = 3                              # (of the third sequence: does not begin at its root)
    elif refused == "accepted":
        accepted[2] = 5
    elif refused == "count":
        m.dev["lens"][m.slot[2]] = m.lens[m.slot[2]] = 4
    elif refused == "slot":
        m.dev["seqs"][2] = 77
    new = torch.full_like(m.dev["lens"], -9)
    m.run(path, accepted, new_lens=new)
    assert psa.psa_last_issued()[0] == (psa.OK if refused is None else psa.ERR_SHAPE)
    skip = () if refused is None else (2,)
    pool, lens = m.want(skip)
    assert torch.equal(m.dev["pool"].cpu(), pool) and torch.equal(m.dev["lens"].cpu(), m.lens)
    listed = [s for b, s in enumerate(m.slot) if not (refused == "slot" and b == 2)]
    assert new.cpu().tolist() == [int(lens[s]) if s in listed else -9 for s in range(len(lens))]


@pytest.mark.gpu
def test_no_rows_at_all():
    m = _made([30, 20], [0, 0], 2, 64, 16, 1, 5)
    new = torch.full_like(m.dev["lens"], -9)
    m.run(new_lens=new)
    assert psa.psa_last_issued()[0] == psa.OK
    assert new.cpu().tolist() == [int(m.lens[s]) if s in m.slot else -9 for s in range(len(m.lens))] and torch.equal(m.dev["pool"].cpu(), m.pool)
    m.run()
    assert torch.equal(m.dev["lens"].cpu(), m.lens)


@pytest.mark.parametrize("change,want", [(dict(seqs=None), "NULL"), (dict(starts=None), "NULL"), (dict(accepted=None), "NULL"), (dict(new_lens=P + 66), "ALIGN"), (dict(n=0), None),
                                         (dict(new_lens=P, seqs=None), None), (dict(new_lens=None), None)])
def test_refusals_without_rows(change, want):
    """Nothing to do but where lengths go elsewhere, and then with all that is read."""
    build.build()
    a = dict(seqs=P, starts=P, accepted=P, n=3, new_lens=P + 64)
    a.update(change)
    cache = psa.Cache(P, P, P, 4, 2, 3, 16, 2, 64)
    assert psa.lib().psa_cache_keep(ctypes.byref(cache), 2, a["seqs"], a["starts"], None, a["accepted"], a["n"], 0, a["new_lens"], None) == (psa.OK if want is None else getattr(psa, "ERR_" + want))
