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


@pytest.mark.parametrize("n", [1, 66])
def test_as_many_tokens_as_a_table_may_hold(n):
    """2^31 - 16 tokens: the columns of the table name one page over and over, whose tokens carry next to no weight, and at the end another.  66 rows of them have more steps than
    32 bits count."""
    d, page, width = 32, 16, (1 << 27) - 1
    tables = torch.zeros(1, width, dtype=torch.int32, device="cuda")
    tables[0, -1] = 1
    g = torch.Generator().manual_seed(8)
    K, V = torch.randn(32, 1, d, generator=g) * 0.1, torch.randn(32, 1, d, generator=g)
    K[:16] -= 100 * d ** -0.5
    K, V = K.to(BF), V.to(BF)
    pool = torch.zeros(2, psa.psa_cache_page_bytes(1, page, d), dtype=torch.uint8, device="cuda")
    zero = torch.zeros(n, dtype=torch.int32, device="cuda")
    two = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    psa.psa_cache_append(K.cuda(), V.cuda(), pool, two, torch.tensor([32], dtype=torch.int32, device="cuda"), zero[:1], ref.starts([32]), page)
    k, v = (ref.held(*ref.quantise(x)) for x in (K, V))
    Q, lse = torch.ones(n, 2, d, dtype=BF, device="cuda"), torch.empty(n, 2, device="cuda")
    out = psa.psa_cache_attention(Q, pool, tables, torch.tensor([width * page], dtype=torch.int32, device="cuda"), zero, ref.starts([1] * n), 1, page, lse=lse)
    assert psa.psa_last_issued()[0] == psa.OK
    # (weights of e^-100: 2^31 of them are 10^-34)
    ref.close(out[:1], lse[:1], ref.attend(Q[:1], k[16:], v[16:], d ** -0.5), BF, 16, 2 * 2.0 ** -11 + ref.UNIT[BF])
    assert (out == out[0]).all() and (lse == lse[0]).all()
