"""psa_cache_attention does not mind how many tokens the tables have room for, only how many are held."""
import pytest
import torch

import serving_reference as ref
from paper_2012_01114_b200 import binding as psa
from test_gpu_cache import Made, _queries

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("lens,q,G,Hkv,d", [([300, 40, 17], [300, 40, 17], 8, 2, 64), ([100] * 64, [64] * 64, 16, 8, 32), ([5000, 3], [1, 1], 4, 2, 128), ([200] * 500, [1] * 500, 4, 8, 32)])
def test_wide_tables(lens, q, G, Hkv, d):
    """Room for 2^20 tokens and for 2^28; the same bits as over a table that fits."""
    c = Made(lens, Hkv, d, 16, 31)
    Q = _queries(sum(q), Hkv * G, d, BF, 4)
    want = c.attend(Q, q, max_q=max(q))
    assert psa.psa_last_issued()[0] == psa.OK
    rows = [(0, min(q[0], 3)), (sum(q[:-1]), 1)]
    for i, (at, n) in zip((0, -1), rows):
        first = len(c.k[i]) - q[i]
        ref.close(want[at:at + n], None, ref.attend(Q[at:at + n], c.k[i][:first + n], c.v[i][:first + n], d ** -0.5), BF, len(c.k[i]), 2 * 2.0 ** -11 + ref.UNIT[BF])
    for width in (1 << 16, 1 << 24) if len(lens) < 4 else (1 << 16,):
        tables = torch.full((c.tables.shape[0], width), -1, dtype=torch.int32, device="cuda")
        tables[:, :c.tables.shape[1]] = c.tables
        got = psa.psa_cache_attention(Q, c.pool, tables, c.lens, c.seqs, ref.starts(q), Hkv, 16, max_q=max(q))
        assert psa.psa_last_issued()[0] == psa.OK and torch.equal(got, want)
