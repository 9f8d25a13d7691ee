"""psa_cache_append_rotary: turned queries against their definition (angles in 80 bits), the cache's bytes against psa_cache_append of turned keys and against the reference's grid.

Errors of a turned number, of amplitude (|a| + |b|): sine and cosine 2^-23 (angle to 2^-25 of half a turn, pi 2^-25 < 2^-23, the functions' own last places in it) and three roundings
of 2^-24, less than 2^-21 altogether; then half a step of the type."""
import random

import pytest
import torch

import drafts_reference as ref
import serving_reference as sref
from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def _freqs(rot, base=10000.0):
    return base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)


class Made:
    """Slots with pages by chance; every sequence holds `old` tokens and gets `new` ones.  The pool's bytes are by chance too, so that a stray write shows."""

    def __init__(self, new, old, H, Hkv, d, page, dtype, seed=0):
        r, g = random.Random(seed), torch.Generator().manual_seed(seed)
        held = [a + b for a, b in zip(new, old)]
        need = [-(-h // page) for h in held]
        self.pages, width, slots = sum(need) + 2, max(need + [1]) + 1, len(new) + 1
        order, self.slot = list(range(self.pages)), list(range(slots))
        r.shuffle(order)
        r.shuffle(self.slot)
        self.slot = self.slot[:len(new)]
        tables, lens = torch.full((slots, width), -1, dtype=torch.int32), torch.zeros(slots, dtype=torch.int32)
        for s, n, m in zip(self.slot, held, need):
            tables[s, :m] = torch.tensor([order.pop() for _ in range(m)], dtype=torch.int32)
            lens[s] = n
        self.new, self.old, self.H, self.Hkv, self.d, self.page, self.rows = new, old, H, Hkv, d, page, sum(new)
        self.tables, self.lens, self.seqs = tables.cuda(), lens.cuda(), torch.tensor(self.slot, dtype=torch.int32, device="cuda")
        self.starts = sref.starts(new)
        self.pool = torch.randint(0, 256, (self.pages, Hkv * page * d * 5 // 4), dtype=torch.uint8, generator=g).cuda()
        qkv = torch.randn(self.rows, H + 2 * Hkv, d, generator=g).to(dtype).cuda()
        self.Q, self.K, self.V = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]

    def append(self, freqs, pool=None, **kw):
        return psa.psa_cache_append_rotary(kw.pop("K", self.K), kw.pop("V", self.V), self.pool if pool is None else pool, self.tables, self.lens, self.seqs, self.starts, self.page, freqs, **kw)

    def positions(self, depths=None):
        base = [o for o, n in zip(self.old, self.new) for _ in range(n)]
        inside = [i for n in self.new for i in range(n)] if depths is None else depths.tolist()
        return [a + b for a, b in zip(base, inside)]


def _check_queries(got, x, positions, freqs, interleaved, amplitude=1.0):
    want, size = ref.turned(x, positions, freqs, interleaved, amplitude)
    tol = sref.UNIT[x.dtype] * want.abs() + 2.0 ** -21 * size + (2.0 ** -25 if x.dtype == HF else 0)
    assert ((got.cpu().double() - want).abs() <= tol).all(), float(((got.cpu().double() - want).abs() / tol).max())


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("H,Hkv,d,rot,page", [(2, 1, 32, 32, 16), (8, 2, 64, 64, 16), (3, 3, 64, 24, 32), (12, 3, 96, 96, 48), (6, 2, 96, 40, 16), (32, 8, 128, 128, 64), (5, 1, 128, 64, 16), (4, 2, 256, 256, 16),
                                              (1, 1, 256, 8, 16)])
def test_queries_and_bytes(H, Hkv, d, rot, page, interleaved, dtype):
    new, old = [1, 5, 0, 18, 2], [0, 300, 7, 15, 4000]
    m = Made(new, old, H, Hkv, d, page, dtype, d + rot)
    freqs = _freqs(rot)
    for depths in (None, torch.randint(0, 6, (m.rows,), dtype=torch.int32, generator=torch.Generator().manual_seed(1)).cuda()):
        pool, again = m.pool.clone(), m.pool.clone()
        k_held, v_held = (torch.empty(m.rows, Hkv, d, dtype=dtype, device="cuda") for _ in range(2))
        k2, v2 = torch.empty_like(k_held), torch.empty_like(v_held)
        out = m.append(freqs, pool, Q=m.Q, depths=depths, interleaved=interleaved, k_held=k_held, v_held=v_held)
        assert psa.psa_last_issued()[0] == psa.OK
        _check_queries(out, m.Q, m.positions(depths), freqs, interleaved)
        turned = m.append(freqs, m.pool.clone(), Q=m.K, depths=depths, interleaved=interleaved)                # (the keys as queries)
        _check_queries(turned, m.K, m.positions(depths), freqs, interleaved)
        psa.psa_cache_append(turned, m.V, again, m.tables, m.lens, m.seqs, m.starts, page, k_held=k2, v_held=v2)
        assert torch.equal(pool, again) and torch.equal(k_held, k2) and torch.equal(v_held, v2)
        assert torch.equal(k_held.cpu(), sref.held(*sref.quantise(turned.cpu())).to(dtype))


def test_other_bytes_stay():
    m = Made([3, 1], [14, 40], 4, 2, 64, 16, BF, 3)
    before = m.pool.clone()
    m.append(_freqs(64))
    mine = torch.zeros_like(before, dtype=torch.bool).cpu()
    for s, n, o in zip(m.slot, m.new, m.old):
        for pos in range(o, o + n):
            page = int(m.tables[s, pos // 16])
            for h in range(2):
                mine[page, ref.byte_places(16, 2, 64, h, pos % 16)] = True
    assert torch.equal(m.pool.cpu()[~mine], before.cpu()[~mine]) and not torch.equal(m.pool, before)


@pytest.mark.parametrize("base", [0, 131072, (1 << 31) - 60, -(1 << 31)])
def test_far_positions(base):
    """Depths up to both ends of 32 bits.  A frequency is rounded to 2^-54 of itself, so that an angle at 2^31 is off by 2^-23 more."""
    m = Made([40], [9], 2, 1, 64, 16, HF, 5)
    freqs, depths = _freqs(64), (torch.arange(40) + base).clamp(max=(1 << 31) - 1).int().cuda()
    out = m.append(freqs, Q=m.Q, depths=depths)
    want, size = ref.turned(m.Q, m.positions(depths), freqs, False)
    assert ((out.cpu().double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -20 * size + 2.0 ** -25).all()


def test_amplitude_and_large_frequencies():
    m = Made([30], [100], 4, 2, 64, 16, HF, 6)
    for freqs, amplitude in ((_freqs(64) / 8, 1.2079), (torch.linspace(-9, 50, 32, dtype=torch.float64, device="cuda"), 0.5), (torch.zeros(16, dtype=torch.float64, device="cuda"), -1.0)):
        _check_queries(m.append(freqs, Q=m.Q, amplitude=amplitude), m.Q, m.positions(), freqs, False, float(torch.tensor(amplitude, dtype=torch.float32)))


@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place(interleaved):
    m = Made([17, 4], [3, 60], 8, 8, 128, 16, BF, 7)
    Q, K, V = (x.contiguous() for x in (m.Q, m.K, m.V))
    pool = m.pool.clone()
    k_held, v_held = torch.empty_like(K), torch.empty_like(V)
    want = m.append(_freqs(96), Q=Q, interleaved=interleaved, k_held=k_held, v_held=v_held)
    got = psa.psa_cache_append_rotary(K, V, pool, m.tables, m.lens, m.seqs, m.starts, 16, _freqs(96), Q=Q, interleaved=interleaved, q_out=Q, k_held=K, v_held=V)
    assert got.data_ptr() == Q.data_ptr() and torch.equal(Q, want) and torch.equal(K, k_held) and torch.equal(V, v_held) and torch.equal(pool, m.pool)


def test_many_rows_and_sequences():
    r = random.Random(8)
    new = [r.choice([0, 1, 1, 2, 9]) for _ in range(700)]
    m = Made(new, [r.randrange(40) for _ in new], 4, 1, 64, 16, BF, 8)
    freqs = _freqs(64)
    _check_queries(m.append(freqs, Q=m.Q), m.Q, m.positions(), freqs, False)
    m = Made([5000], [0], 20, 4, 128, 64, BF, 9)      # heads shared out, several a thread
    freqs = _freqs(128)
    _check_queries(m.append(freqs, Q=m.Q), m.Q, m.positions(), freqs, False)


def test_places_that_do_not_exist():
    """An unknown slot, a page that is missing and a table that ends: reported, and what has a place is written; rows behind the last sequence are left as they are."""
    m = Made([2, 3, 2], [15, 20, 5], 4, 2, 64, 16, BF, 10)
    freqs = _freqs(64)
    good = m.pool.clone()
    want = m.append(freqs, good, Q=m.Q)
    m.seqs[0] = 99
    out = torch.full((m.rows + 2, 4, 64), 7.0, dtype=BF, device="cuda")
    Q, K, V = (torch.cat([x, x[:2]]) for x in (m.Q, m.K, m.V))
    pool = m.pool.clone()
    psa.psa_cache_append_rotary(K, V, pool, m.tables, m.lens, m.seqs, m.starts, 16, freqs, Q=Q, q_out=out)
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
    assert torch.equal(out[2:7], want[2:]) and (out[:2] == 7).all() and (out[7:] == 7).all()
    same = (pool == m.pool).all(-1) | (pool == good).all(-1)
    assert same.all() and not torch.equal(pool, m.pool)


def test_without_queries_and_with_nan():
    m = Made([4], [30], 4, 2, 64, 16, BF, 11)
    a, b = m.pool.clone(), m.pool.clone()
    assert m.append(_freqs(64), a) is None
    m.append(_freqs(64), b, Q=m.Q)
    assert torch.equal(a, b)
    K = m.K.clone()
    K[1, 0, 5] = float("nan")                    # its partner is channel 37: both groups of the token's head are NaN, and nothing else
    k_held = torch.empty(4, 2, 64, dtype=BF, device="cuda")
    clean = torch.empty_like(k_held)
    m.append(_freqs(64), b, K=K, k_held=k_held)
    m.append(_freqs(64), a, k_held=clean)
    nan = torch.isnan(k_held)
    assert nan[1, 0].all() and nan.sum() == 64 and torch.equal(k_held[~nan], clean[~nan])


def test_captured_and_on_another_stream():
    m = Made([1, 1, 1], [5, 100, 63], 8, 2, 128, 64, BF, 12)
    freqs, s = _freqs(128), torch.cuda.Stream()
    out = torch.empty(3, 8, 128, dtype=BF, device="cuda")
    want = m.append(freqs, Q=m.Q).clone()
    pool = m.pool.clone()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        m.append(freqs, Q=m.Q, q_out=out)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(pool, m.pool)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.append(freqs, Q=m.Q, q_out=out)
        m.append(freqs, Q=m.Q, q_out=out)
    for _ in range(2):
        out.zero_()
        m.pool.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
