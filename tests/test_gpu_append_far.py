"""psa_cache_append_rotary at the far end of 32 bits with frequencies of all sizes: the tolerance is that of near positions (tests/test_gpu_append_rotary.py), since the angle is formed in 64 bits.  With
2^31 positions a frequency's fraction of a turn has to be good to 2^-58: an angle off by more than 2^-23 shows in channels that nearly cancel."""
import pytest
import torch

from paper_2012_01114_b200 import binding as psa
from test_gpu_append_rotary import Made, _check_queries, _freqs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("what", ["usual", "up to 50", "up to 3000", "below 1e-9"])
@pytest.mark.parametrize("base", [0, (1 << 31) - 2000, -(1 << 31)])
def test_angles_at_far_positions(base, what, interleaved):
    m = Made([700], [9], 16, 1, 64, 16, torch.float16, 5)
    freqs = {"usual": _freqs(64), "up to 50": torch.linspace(-9, 50, 32, dtype=torch.float64, device="cuda"), "up to 3000": 3000 * _freqs(64, 1e6),
             "below 1e-9": 1e-9 * _freqs(64)}[what]
    depths = (torch.arange(700) * (2 if base > 0 else 1) + base).clamp(max=(1 << 31) - 1).int().cuda()
    out = m.append(freqs, Q=m.Q, depths=depths, interleaved=interleaved)
    _check_queries(out, m.Q, m.positions(depths), freqs, interleaved)
    pool, again = m.pool.clone(), m.pool.clone()
    turned = m.append(freqs, pool, Q=m.K, depths=depths, interleaved=interleaved)            # (the keys as queries: the cache holds the same)
    psa.psa_cache_append(turned, m.V, again, m.tables, m.lens, m.seqs, m.starts, 16)
    assert torch.equal(pool, again)
    _check_queries(turned, m.K, m.positions(depths), freqs, interleaved)
