"""The paged cache in 4 bits: what psa_cache_append writes, byte by byte, and psa_cache_attention against attention over the held values in 64 bits.  Rounded on the
way to an output: the weight and the held value to fp16 (2^-11 each), the result to its type (tests/serving_reference.py)."""
import pytest
import torch

import serving_reference as ref
from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


class Made:
    """A cache filled by the reference's own layout code, pages in the order of chance, everything behind a sequence's end set to 0xff (NaN in every scale)."""

    def __init__(self, lens, Hkv, d, page, seed=0, spare=2, extra_slots=1):
        g = torch.Generator().manual_seed(seed)
        need = [-(-n // page) for n in lens]
        slots, width = len(lens) + extra_slots, max(need + [1]) + 1
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=g).tolist()
        self.tables = torch.full((slots, width), -1, dtype=torch.int32)
        pool = torch.full((self.pages, Hkv, page // 16, 20 * d), 255, dtype=torch.uint8)
        self.k, self.v, self.slot = [], [], torch.randperm(slots, generator=g)[:len(lens)].tolist()
        length = torch.zeros(slots, dtype=torch.int32)
        for s, n, m in zip(self.slot, lens, need):
            mine = [order.pop() for _ in range(m)]
            self.tables[s, :m] = torch.tensor(mine, dtype=torch.int32)
            length[s] = n
            up = -(-n // 16) * 16
            k, v = (torch.randn(up, Hkv, d, generator=g).clamp(-4, 4) + (torch.randn(1, Hkv, d, generator=g) if i == 0 else 0) for i in range(2))
            kq, vq = ref.quantise(k), ref.quantise(v)
            for q in (kq, vq):          # (tokens behind the end: NaN scales, full codes)
                q[0][n:], q[1][n:], q[2][n:] = 15, float("nan"), float("nan")
            for h in range(Hkv if up else 0):
                img = ref.block_images([x[:, h].contiguous() for x in kq], [x[:, h].contiguous() for x in vq], up)
                for b in range(up // 16):
                    pool[mine[b * 16 // page], h, b * 16 % page // 16] = img[b]
            self.k.append(ref.held(*(x[:n] for x in kq)))
            self.v.append(ref.held(*(x[:n] for x in vq)))
        self.pool, self.tables, self.lens = pool.view(self.pages, -1).cuda(), self.tables.cuda(), length.cuda()
        self.seqs = torch.tensor(self.slot, dtype=torch.int32, device="cuda")
        self.Hkv, self.d, self.page = Hkv, d, page

    def attend(self, Q, q, **kw):
        return psa.psa_cache_attention(Q, self.pool, self.tables, self.lens, self.seqs, ref.starts(q), self.Hkv, self.page, **kw)


def _queries(rows, H, d, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(rows, H, d, device="cuda").normal_(generator=g).to(dtype)


def _check(c, q, G, dtype, max_q=None, scale=None, Q=None):
    H = c.Hkv * G
    Q = _queries(sum(q), H, c.d, dtype, 3) if Q is None else Q
    lse = torch.full((sum(q), H), float("nan"), device="cuda")
    out = c.attend(Q, q, max_q=max(q + [1]) if max_q is None else max_q, lse=lse, scale=scale)
    assert psa.psa_last_issued()[0] == psa.OK
    at = 0
    for n, k, v in zip(q, c.k, c.v):
        if n:
            r = ref.attend(Q[at:at + n], k, v, c.d ** -0.5 if scale is None else scale)
            ref.close(out[at:at + n], lse[at:at + n], r, dtype, len(k), 2 * 2.0 ** -11 + ref.UNIT[dtype])
        at += n
    return out


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("G,Hkv,d,page", [(1, 2, 32, 16), (1, 1, 64, 64), (4, 2, 128, 16), (8, 1, 128, 64), (3, 3, 96, 48), (8, 2, 256, 32), (9, 1, 64, 16), (20, 1, 128, 32), (64, 1, 64, 128)])
def test_single_tokens(G, Hkv, d, page, dtype):
    lens = [1, 15, 16, 17, 64, 200, 0, 333]
    _check(Made(lens, Hkv, d, page, d), [1] * len(lens), G, dtype)


@pytest.mark.parametrize("d", [32, 64, 96, 128, 256])
def test_several_queries(d):
    """Also more of them than tokens are held (the first rows see nothing), none at all, and a bound that is too small."""
    lens, q = [5, 40, 100, 3, 0, 31], [5, 3, 0, 7, 2, 20]
    c = Made(lens, 2, d, 16, 7)
    a = _check(c, q, 3, BF)
    b = _check(c, q, 3, BF, max_q=1)
    assert torch.allclose(a.float(), b.float(), atol=3e-2)


@pytest.mark.parametrize("lens,Hkv,d", [([20000], 1, 64), ([9000, 1, 40], 2, 128), ([1] * 300, 1, 64), ([130, 2000] * 80, 1, 32)])
def test_split_rows_and_many_sequences(lens, Hkv, d):
    c = Made(lens, Hkv, d, 64, 11)
    q = [1] * len(lens)
    a = _check(c, q, 4, BF)
    for _ in range(3):                  # whoever joins the parts of a row, the result is the same
        assert torch.equal(a, _check(c, q, 4, BF))


def test_scale_strides_and_small_numbers():
    c = Made([50, 70], 2, 64, 16, 12)
    _check(c, [1, 1], 4, BF, scale=0.9)
    buf = _queries(3, 20, 64, BF, 5)
    _check(c, [1, 2], 4, BF, Q=buf[:, 4:12])
    for size in (1e-30, 1e-6, 1e6):     # bf16 queries beyond what fp16 holds: rows are scaled by a power of two
        _check(c, [1, 1], 4, BF, Q=(_queries(2, 8, 64, BF, 6) * size).to(BF), scale=0.125 / size)


def test_a_nan_is_seen_by_those_that_see_it():
    """Three queries, the last token's values NaN: only the last query has it.  A NaN among the keys likewise."""
    for which in (0, 1):
        c = Made([40], 1, 64, 16, 13)
        K, V = (torch.randn(1, 1, 64, device="cuda").to(BF) for _ in range(2))
        plain = c.attend(_queries(3, 2, 64, BF), [3], max_q=3).clone()
        (K, V)[which][0, 0, 40] = float("nan")
        psa.psa_cache_append(K, V, c.pool, c.tables, c.lens, c.seqs, ref.starts([1]), 16)
        out = c.attend(_queries(3, 2, 64, BF), [3], max_q=3)
        assert torch.equal(out[:2], plain[:2])
        got = torch.isnan(out[2].view(2, 64))
        assert got.all() if which == 0 else (got[:, 32:].all() and not got[:, :32].any())


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("Hkv,d,page", [(1, 32, 16), (3, 64, 32), (2, 96, 16), (2, 128, 64), (1, 256, 16)])
def test_append_writes_its_bytes_and_no_others(Hkv, d, page, dtype):
    old, new = [0, 5, 31, 16, 0, 7], [1, 2, 40, 0, 33, 1]
    c = Made([a + b for a, b in zip(old, new)], Hkv, d, page, 21)
    rows = sum(new)
    buf = torch.randn(rows, 2 * Hkv + 1, d, generator=torch.Generator().manual_seed(4)).to(dtype)
    buf[0, 0, :32], buf[1, 0, 3] = 0.5, 1e5 if dtype == BF else 6e4                  # a constant group, a number beyond the grid
    buf[2, 0, :32] *= 1e-6
    K, V = buf[:, :Hkv].cuda(), buf.cuda()[:, Hkv + 1:]
    want = c.pool.cpu().clone()
    kq, vq = ref.quantise(K.cpu()), ref.quantise(V.cpu())
    at = 0
    for s, a, b in zip(c.slot, old, new):
        for i in range(b):
            pos = a + i
            page_id = int(c.tables[s, pos // page])
            for h in range(Hkv):
                ref.put(want[page_id], h, page, d, pos % page, [x[at + i, h] for x in kq], [x[at + i, h] for x in vq])
        at += b
    k_held, v_held = torch.empty(rows, Hkv, d, dtype=dtype, device="cuda"), torch.empty(rows, Hkv, d, dtype=dtype, device="cuda")
    psa.psa_cache_append(buf.cuda()[:, :Hkv], V, c.pool, c.tables, c.lens, c.seqs, ref.starts(new), page, k_held=k_held, v_held=v_held)
    assert psa.psa_last_issued()[0] == psa.OK
    assert torch.equal(c.pool.cpu(), want)
    assert torch.equal(k_held.cpu(), ref.held(*kq).float().to(dtype)) and torch.equal(v_held.cpu(), ref.held(*vq).float().to(dtype))
    # half a step of the grid, and what rounding S and M to fp16 costs at its ends: at most 16 + 1 halves of 2^-10 of |S| + |lo|
    x, S, M = K.cpu().float().clamp(-20000, 20000), kq[1].double(), kq[2].double()
    err = (ref.held(*kq) - x.double()).abs().unflatten(-1, (-1, 32)).amax(-1)
    assert (err <= S / 32 * 1.001 + 2.0 ** -10 * (S + M.abs()) + 1e-7).all()
    psa.psa_cache_append(buf.cuda()[:, :Hkv].contiguous(), V, c.pool, c.tables, c.lens, c.seqs, ref.starts(new), page)      # without the held values
    assert torch.equal(c.pool.cpu(), want)


def test_append_of_what_is_no_number():
    c = Made([3], 1, 64, 16, 22)
    K = torch.randn(3, 1, 64, device="cuda").to(BF)
    V = K.clone()
    K[0, 0, 5], K[1, 0, 40], V[2, 0, 7] = float("nan"), float("inf"), float("-inf")
    k, v = torch.empty_like(K), torch.empty_like(V)
    psa.psa_cache_append(K, V, c.pool, c.tables, c.lens, c.seqs, ref.starts([3]), 16, k_held=k, v_held=v)
    assert torch.isnan(k[0, 0, :32]).all() and torch.isfinite(k[0, 0, 32:]).all() and torch.isfinite(k[1:]).all() and torch.isfinite(v).all()
    assert abs(float(k[1, 0, 40]) - 20000) < 200 and abs(float(v[2, 0, 7]) + 20000) < 200


def test_append_then_attend_in_steps():
    """A prompt of 20 tokens and then 30 single ones, each step against all tokens so far; in place of the held values, k and v themselves."""
    Hkv, d, page, G = 2, 64, 16, 4
    tables = torch.tensor([[3, 0, 2, 1]], dtype=torch.int32, device="cuda")
    lens, seqs = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    pool = torch.full((4, psa.psa_cache_page_bytes(Hkv, page, d)), 255, dtype=torch.uint8, device="cuda")
    ks, vs = [], []
    for step in range(31):
        n = 20 if step == 0 else 1
        K, V, Q = _queries(n, Hkv, d, BF, 3 * step), _queries(n, Hkv, d, BF, 3 * step + 1), _queries(n, Hkv * G, d, BF, 3 * step + 2)
        lens += n
        kq, vq = ref.quantise(K.cpu()), ref.quantise(V.cpu())
        ks.append(ref.held(*kq)); vs.append(ref.held(*vq))
        psa.psa_cache_append(K, V, pool, tables, lens, seqs, ref.starts([n]), page, k_held=K, v_held=V)
        assert torch.equal(K.cpu(), ks[-1].float().to(BF))
        out = psa.psa_cache_attention(Q, pool, tables, lens, seqs, ref.starts([n]), Hkv, page, max_q=n)
        ref.close(out, None, ref.attend(Q, torch.cat(ks), torch.cat(vs), d ** -0.5), BF, 50, 2 * 2.0 ** -11 + ref.UNIT[BF])


def test_places_that_do_not_exist():
    c = Made([40, 20], 1, 64, 16, 23)
    Q, K = _queries(2, 2, 64, BF), torch.zeros(2, 1, 64, dtype=BF, device="cuda")
    want = _check(c, [1, 1], 2, BF, Q=Q)
    before = c.pool.clone()
    slot = c.slot[0]
    page = c.tables[slot, 1].clone()
    for bad in (-1, c.pages, 1 << 30):
        c.tables[slot, 1] = bad
        out = c.attend(Q, [1, 1])
        assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
        assert torch.isfinite(out).all() and torch.equal(out[1], want[1])
        c.tables[slot, 1] = page
        c.tables[slot, 2], keep = bad, c.tables[slot, 2].clone()
        psa.psa_cache_append(K[:1], K[:1], c.pool, c.tables, c.lens, c.seqs[:1], ref.starts([1]), 16)
        assert psa.psa_last_issued()[0] == psa.ERR_SHAPE and torch.equal(c.pool, before)
        c.tables[slot, 2] = keep
    for bad in (-1, c.tables.shape[0], 1 << 30):
        seqs = c.seqs.clone()
        seqs[0] = bad
        out = psa.psa_cache_attention(Q, c.pool, c.tables, c.lens, seqs, ref.starts([1, 1]), 1, 16)
        assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
        assert (out[0] == 0).all() and torch.equal(out[1], want[1])
    lens = c.lens.clone()
    lens[slot] = 1 << 30                # longer than the table
    psa.psa_cache_attention(Q, c.pool, c.tables, lens, c.seqs, ref.starts([1, 1]), 1, 16)
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE
    assert torch.equal(_check(c, [1, 1], 2, BF, Q=Q), want)


def test_another_stream_and_graph_replay():
    c = Made([100, 3000], 2, 64, 16, 24)
    Q = _queries(2, 8, 64, BF)
    starts = ref.starts([1, 1])
    call = lambda **kw: psa.psa_cache_attention(Q, c.pool, c.tables, c.lens, c.seqs, starts, 2, 16, **kw)  # noqa: E731
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = call(stream=s)
    s.synchronize()
    assert torch.equal(want, got)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out=out)
    for n in (2999, 17, 3000):
        c.lens[c.slot[1]] = n
        graph.replay()
        graph.replay()
        assert torch.equal(out.clone(), call())


def test_offsets_beyond_32_bits():
    """A pool of 5 GB, the sequence's pages at its end."""
    Hkv, d, page = 8, 128, 128
    size = psa.psa_cache_page_bytes(Hkv, page, d)
    pages = (5 << 30) // size
    small = Made([300, 130], Hkv, d, page, 25)
    pool = torch.empty(pages, size, dtype=torch.uint8, device="cuda")
    pool[pages - small.pages:] = small.pool
    tables = torch.where(small.tables >= 0, small.tables + pages - small.pages, small.tables)
    Q = _queries(2, 32, d, BF)
    want = small.attend(Q, [1, 1])
    got = psa.psa_cache_attention(Q, pool, tables, small.lens, small.seqs, ref.starts([1, 1]), Hkv, page)
    assert psa.psa_last_issued()[0] == psa.OK and torch.equal(got, want)
    K, V = _queries(2, Hkv, d, BF, 1), _queries(2, Hkv, d, BF, 2)
    psa.psa_cache_append(K, V, pool, tables, small.lens, small.seqs, ref.starts([1, 1]), page)
    psa.psa_cache_append(K, V, small.pool, small.tables, small.lens, small.seqs, ref.starts([1, 1]), page)
    assert torch.equal(pool[pages - small.pages:], small.pool)


def test_starts_that_descend():
    c = Made([40, 20, 30], 1, 64, 16, 26)
    Q = _queries(9, 2, 64, BF)
    bad = torch.tensor([0, 9, 0, 9], dtype=torch.int32, device="cuda")
    out = psa.psa_cache_attention(Q, c.pool, c.tables, c.lens, c.seqs, bad, 1, 16, max_q=9, out=torch.full((9, 128), 3.0, dtype=BF, device="cuda"))
    assert psa.psa_last_issued()[0] == psa.ERR_SHAPE and (out == 3).all()
    far = torch.tensor([-3, 4, 4, 1000], dtype=torch.int32, device="cuda")               # rows outside the tensor are not touched
    assert torch.equal(psa.psa_cache_attention(Q, c.pool, c.tables, c.lens, c.seqs, far, 1, 16, max_q=9), c.attend(Q, [4, 0, 5], max_q=9))
    assert psa.psa_last_issued()[0] == psa.OK


def test_more_sequences_than_a_launch_takes():
    lens = [(i * 37) % 70 for i in range(700)]
    c = Made(lens, 1, 32, 16, 27)
    _check(c, [i % 3 for i in range(700)], 2, BF)


def test_calls_in_a_row_in_one_graph():
    """Each call of a graph has a status and work counter of its own, clear at every replay, whatever ran in between; other calls of the library among them."""
    c = Made([100, 3000], 2, 64, 16, 29)
    starts = ref.starts([70, 130])
    Q, K, V = _queries(200, 8, 64, BF), _queries(200, 2, 64, BF, 1), _queries(200, 2, 64, BF, 2)
    Q1, one = _queries(2, 8, 64, BF, 4), ref.starts([1, 1])
    X = _queries(1, 256, 128, BF, 5).view(1, 256, 2, 64)
    outs = [torch.empty(200, 512, dtype=BF, device="cuda") for _ in range(3)] + [torch.empty(2, 512, dtype=BF, device="cuda") for _ in range(3)]

    def calls():
        psa.psa_prompt_attention(Q, K, V, starts, out=outs[0])
        psa.psa_prompt_attention(Q, K, V, starts, out=outs[1])
        psa.psa_cache_attention(Q1, c.pool, c.tables, c.lens, c.seqs, one, 2, 16, out=outs[3])
        psa.psa_attention_core(X, X, X, psa.MASKED)
        psa.psa_prompt_attention(Q, K, V, starts, out=outs[2])
        psa.psa_cache_attention(Q1, c.pool, c.tables, c.lens, c.seqs, one, 2, 16, out=outs[4])
        psa.psa_cache_attention(Q1, c.pool, c.tables, c.lens, c.seqs, one, 2, 16, out=outs[5])

    calls()
    want = [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    place = c.tables[c.slot[1], 3].clone()
    for bad in (False, True, False, True, True, False):
        c.tables[c.slot[1], 3] = -1 if bad else place
        for o in outs:
            o.fill_(7)
        graph.replay()
        assert psa.psa_last_issued()[0] == (psa.ERR_SHAPE if bad else psa.OK)
        if not bad:
            assert all(torch.equal(a, b) for a, b in zip(outs, want))
        graph.replay()
        torch.cuda.synchronize()
        c.tables[c.slot[1], 3] = place
        psa.psa_cache_attention(Q1, c.pool, c.tables, c.lens, c.seqs, one, 2, 16)
        assert psa.psa_last_issued()[0] == psa.OK
        with torch.cuda.graph(graph := torch.cuda.CUDAGraph()):        # (a capture of its own starts clear as well)
            calls()


@pytest.mark.parametrize("d,longest,n", [(128, 32, 120), (128, 70, 160), (64, 300, 90), (96, 6, 87), (256, 150, 90), (128, 900, 60), (128, 6000, 30), (64, 3000, 36)])
def test_batches_of_about_as_many_rows_as_ctas_and_more(d, longest, n):
    """Rows of 1, 2, .. steps, one to a warp or to a CTA by how many there are of each."""
    g = torch.Generator().manual_seed(n)
    lens = [longest] + [int(longest ** float(torch.rand(1, generator=g))) for _ in range(n - 1)]
    _check(Made(lens, 8 if d < 256 else 4, d, 32, 30), [1 + i % 2 for i in range(n)], 2, HF)
