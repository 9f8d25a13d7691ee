"""Rows in which one key outweighs all others by e^gap and carries a value of zero, so that the output is what the others' small weights leave.  A weight is rounded to
16 bits for the second product.  In fp16 it is held at 2^7 times its ratio to the running maximum, which is at most 2^8 behind the largest: rounded to 2^-11 of itself, and below
fp16's normal numbers to 2^-25, which is 2^-32 of a largest weight of 2^7 or more.  Hence a bound of (roundings + 1e-4) sum_j w_ij |v_j| + keys 2^-32 max |v|."""
import pytest
import torch

import serving_reference as ref
from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
GAPS = [0, 5.5, 10, 14, 16, 18]


def _tokens(n, Hkv, d, dtype, gap, at, seed):
    """Keys with scores near zero against a query of ones, but for key `at`, whose score is the gap; values of 500 to 1500, its own zero."""
    g = torch.Generator().manual_seed(seed)
    K, V = torch.randn(n, Hkv, d, generator=g) * 0.05, 500 + 1000 * torch.rand(n, Hkv, d, generator=g)
    K[at], V[at] = gap * d ** -0.5, 0
    return K.to(dtype), V.to(dtype)


def _check(out, lse, Q, k, v, dtype, roundings):
    r, size, r_lse = ref.attend(Q, k, v, Q.shape[2] ** -0.5)
    got = out.detach().cpu().double().view(r.shape)
    tol = (roundings + 1e-4) * size + len(k) * 2.0 ** -32 * 1500 + 2.0 ** -24
    assert ((got - r).abs() <= tol).all(), float(((got - r).abs() / tol).max())
    assert ((lse.cpu().double() - r_lse).abs() <= 5e-5 * (1 + r_lse.abs())).all()


@pytest.mark.parametrize("gap", GAPS)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("nq,nk,H,Hkv,d,at", [(256, 256, 2, 2, 64, 0), (40, 256, 4, 1, 128, 0), (9, 300, 2, 1, 96, 130), (3, 5000, 4, 2, 128, 0), (5, 4000, 4, 2, 64, 2500)])
def test_prompt(nq, nk, H, Hkv, d, at, dtype, gap):
    K, V = _tokens(nk, Hkv, d, dtype, gap, at, nk + d)
    Q = torch.ones(nq, H, d, dtype=dtype)
    lse = torch.empty(nq, H, device="cuda")
    out = psa.psa_prompt_attention(Q.cuda(), K.cuda(), V.cuda(), ref.starts([nq]), ref.starts([nk]), lse=lse)
    assert psa.psa_last_issued()[0] == psa.OK
    _check(out, lse, Q, K, V, dtype, 2 * ref.UNIT[dtype])


@pytest.mark.parametrize("gap", GAPS)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,q,H,Hkv,d,at", [([256], [1], 4, 1, 128, 0), ([256, 40, 31], [1, 1, 1], 2, 2, 64, 3), ([300], [5], 4, 1, 96, 130), ([5000], [1], 4, 2, 128, 0), ([1000], [3], 2, 2, 32, 900),
                                               ([500], [1], 2, 1, 256, 0), ([64] * 300, [1] * 300, 2, 1, 64, 0)])
def test_cache(lens, q, H, Hkv, d, at, dtype, gap):
    page = 32
    made = [_tokens(n, Hkv, d, dtype, gap, at, n + d + i) for i, n in enumerate(lens)]
    need = [-(-n // page) for n in lens]
    tables = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    for i, n in enumerate(need):
        tables[i, :n] = torch.arange(n) + sum(need[:i])
    pool = torch.full((sum(need), psa.psa_cache_page_bytes(Hkv, page, d)), 255, dtype=torch.uint8, device="cuda")
    tables, length, seqs = tables.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.arange(len(lens), dtype=torch.int32, device="cuda")
    psa.psa_cache_append(torch.cat([k for k, _ in made]).cuda(), torch.cat([v for _, v in made]).cuda(), pool, tables, length, seqs, ref.starts(lens), page)
    Q, lse = torch.ones(sum(q), H, d, dtype=dtype), torch.empty(sum(q), H, device="cuda")
    out = psa.psa_cache_attention(Q.cuda(), pool, tables, length, seqs, ref.starts(q), Hkv, page, max_q=max(q), lse=lse)
    assert psa.psa_last_issued()[0] == psa.OK
    first = 0
    for i, n in enumerate(q):
        if i < 3:           # (the sequences of the long batch are alike)
            k, v = (ref.held(*ref.quantise(x)) for x in made[i])
            _check(out[first:first + n], lse[first:first + n], Q[first:first + n], k, v, dtype, 2 * 2.0 ** -11 + ref.UNIT[dtype])
        first += n


@pytest.mark.parametrize("dtype", [BF, HF])
def test_scores_beyond_32_bits_stay_finite(dtype):
    """Scores of 10^8, where neighbouring fp32 numbers are 8 apart: the weights mean little, but nothing overflows."""
    g = torch.Generator().manual_seed(3)
    K, V = (torch.randn(700, 1, 64, generator=g).to(dtype) for _ in range(2))
    Q = torch.randn(40, 4, 64, generator=g).to(dtype)
    out = psa.psa_prompt_attention(Q.cuda(), K.cuda(), V.cuda(), ref.starts([40]), ref.starts([700]), scale=3e6)
    assert torch.isfinite(out).all() and float(out.abs().max()) <= 1.01 * float(V.abs().max())
