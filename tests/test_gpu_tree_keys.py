"""psa_tree_attention over long contexts where rounding a key would show: channels many times the others, and queries so large that a row attends to a few tokens.  Both kernels, against attention over
the held values in 64 bits.

A score may be off by 2^-20 scale sum_c |q_c k_c| (what two fp16 numbers leave of a key, 2^-22 of it, and its sum in 32 bits), which a log-sum-exp then is too; its own exponentials, sums and the factor
from scores to exponents add 2^-20 of the larger of both, and 2e-5 (sums of 10^4 numbers in 32 bits).  A weight is off by twice a score's error, relative; the other roundings of an output as in
test_gpu_tree.py.

The kernel that takes sixteen rows at a time never forms a key: a score is the sum over groups of M_g sum q and S_g sum q (1 + c / 16) in 32 bits, terms that cancel where a channel is large beside
the others of its group.  Two products and two sums a group, each rounded by 2^-24 of what has come together, which is no more than sum_c |q_c| (|M_g| + 2 S_g): 2^-24 of it inside the groups
altogether, as much for every sum of up to three groups (d = 96, 64), four at d = 128 where the largest group decides: less than 2^-22 of it, scaled."""
import random

import pytest
import torch

import drafts_reference as ref
import serving_reference as sref
from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _cache(n, Hkv, d, page, channels, times, g):
    """One sequence of n tokens, some channels of whose keys are `times` as large as the others -> pool, table, K and V as held, |M| + 2 S of the keys' groups."""
    up = -(-n // page) * page
    k, v = torch.randn(up, Hkv, d, generator=g), torch.randn(up, Hkv, d, generator=g).clamp(-4, 4)
    k[:, :, channels] = k[:, :, channels] + times * (1 + torch.rand(1, Hkv, len(channels), generator=g))
    kq, vq = sref.quantise(k), sref.quantise(v)
    pool = torch.stack([sref.block_images([x[:, h].contiguous() for x in kq], [x[:, h].contiguous() for x in vq], up).view(up // page, page // 16, 20 * d) for h in range(Hkv)], 1)
    measure = (kq[2].double().abs() + 2 * kq[1].double())[:n].repeat_interleave(32, -1)
    return pool.reshape(up // page, -1).cuda(), torch.arange(up // page, dtype=torch.int32, device="cuda")[None], sref.held(*(x[:n] for x in kq)), sref.held(*(x[:n] for x in vq)), measure


@pytest.mark.parametrize("form", ["sixteens", "tiles"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("times,size", [(0, 1), (0, 8), (0, 16), (30, 1), (100, 1), (30, 8)])
@pytest.mark.parametrize("n,d,G,Hkv", [(2200, 128, 4, 1), (6000, 64, 2, 2), (3000, 96, 8, 1)])
def test_keys_keep_their_value(n, d, G, Hkv, times, size, dtype, form):
    page, tree = 64, ref.random_tree(20, random.Random(n))[0]
    g = torch.Generator().manual_seed(n + times + size)
    pool, table, k, v, measure = _cache(n, Hkv, d, page, [3, d // 2 + 1, d - 9], times, g)
    if form == "tiles":                          # (by the keys that the table has room for)
        table = torch.nn.functional.pad(table, (0, 65536 // page - table.shape[1]), value=-1)
    Q = (size * torch.randn(20, Hkv * G, d, generator=g)).to(dtype).cuda()
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.full((20, Hkv * G), float("nan"), device="cuda")
    out = psa.psa_tree_attention(Q, pool, table, one + n, one, sref.starts([20]), torch.tensor(tree, dtype=torch.int32, device="cuda"), Hkv, page, 1024 if form == "tiles" else 20, lse=lse)
    assert psa.psa_last_issued()[0] == psa.OK
    want, held, want_lse = ref.attend(Q, k, v, d ** -0.5, ref.seen_by(tree, 20, n))
    q = Q.cpu().double().view(20, Hkv, G, d).abs()
    over = lambda x: d ** -0.5 * torch.einsum("ihgd,jhd->ihgj", q, x).amax(-1).reshape(20, Hkv * G)  # noqa: E731
    score = 2.0 ** -20 * torch.maximum(over(k.abs()), want_lse.abs()) + 2e-5
    if form == "sixteens":
        score += 2.0 ** -22 * over(measure)
    off = (lse.cpu().double() - want_lse).abs()
    assert (off <= score).all(), float((off / score).max())
    tol = (2 * 2.0 ** -11 + UNIT[dtype] + 1e-4 + 2 * score[..., None]) * held + n * 2.0 ** -25 * 4 + 2.0 ** -24
    off = (out.cpu().double().view(want.shape) - want).abs()
    assert (off <= tol).all(), float((off / tol).max())
