"""`starts` of psa_prompt_attention that do not ascend: nothing is computed, and psa_last_issued says so."""
import pytest
import torch

from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu


def _call(q_starts, k_starts=None, rows=50, d=64, dtype=torch.bfloat16, H=2):
    g = torch.Generator(device="cuda").manual_seed(2)
    Q, K, V = (torch.empty(rows, h, d, device="cuda").normal_(generator=g).to(dtype) for h in (H, 1, 1))
    ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out, lse = torch.full((rows, H * d), 3.0, dtype=dtype, device="cuda"), torch.full((rows, H), 3.0, device="cuda")
    psa.psa_prompt_attention(Q, K, V, ints(q_starts), ints(k_starts), out=out, lse=lse)
    return psa.psa_last_issued()[0], out, lse


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q,k", [([0, 50, 0, 50, 0, 50] * 20, None), ([0, 20, 19, 50], None), ([0, 30, 20], [0, 30, 50]), ([0, 30, 50], [0, 50, 30]), ([10, 5], None), ([0, 10, 50], [0, 40, -3]),
                                 ([0, 20, 1 << 30, 50], None), ([0, 50, 0], [0, 1, 2])])
def test_descending(q, k, d):
    status, out, lse = _call(q, k, d=d)
    assert status == psa.ERR_SHAPE and (out == 3).all() and (lse == 3).all()


def test_in_parts():
    """Few rows and many keys, which are cut into parts."""
    status, out, lse = _call([0, 3, 2], [0, 3000, 5000], rows=5000)
    assert status == psa.ERR_SHAPE and (out == 3).all() and (lse == 3).all()


def test_ascending_beyond_the_tensors():
    """Rows that do not exist are none: what is left ascends."""
    status, out, _ = _call([-9, -3, 20, 50, 60, 1000])
    want = _call([0, 0, 20, 50, 50, 50])
    assert status == want[0] == psa.OK and torch.equal(out, want[1])
    assert _call([60, 1 << 30])[0] == psa.OK


def test_only_the_part_in_which_they_descend():
    """600 sequences of a row each; the second launch's descend."""
    starts = list(range(601))
    starts[550], starts[551] = 551, 550
    status, out, _ = _call(starts, rows=600)
    want = _call(list(range(601)), rows=600)[1]
    assert status == psa.ERR_SHAPE and torch.equal(out[:512], want[:512]) and (out[512:] == 3).all()
