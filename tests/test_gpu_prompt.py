"""psa_prompt_attention against its definition in 64 bits.  A weight is rounded once to the storage type and so is an output: two unit roundoffs of
sum_j w_ij |v_j|, and 1e-4 of it for sums and exponentials in 32 bits (tests/serving_reference.py)."""
import math

import pytest
import torch

import serving_reference as ref
from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def _inputs(q, k, H, Hkv, d, dtype, seed=0, fused=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.empty(s, device="cuda").normal_(generator=g).clamp(-4, 4).to(dtype)  # noqa: E731
    if fused:
        rows = rand(sum(q), H + 2 * Hkv, d)
        return rows[:, :H], rows[:, H:H + Hkv], rows[:, H + Hkv:]
    return rand(sum(q), H, d), rand(sum(k), Hkv, d), rand(sum(k), Hkv, d)


def _check(Q, K, V, q, k, scale=None, out=None, lse=None, **kw):
    qs, ks = ref.starts(q), ref.starts(k)
    if lse is None:
        lse = torch.full(Q.shape[:2], float("nan"), device="cuda")
    out = psa.psa_prompt_attention(Q, K, V, qs, ks, scale=scale, lse=lse, out=out, **kw)
    assert psa.psa_last_issued()[0] == psa.OK
    a = b = 0
    for nq, nk in zip(q, k):
        if nq:
            r = ref.attend(Q[a:a + nq], K[b:b + nk], V[b:b + nk], Q.shape[2] ** -0.5 if scale is None else scale)
            ref.close(out[a:a + nq], lse[a:a + nq], r, Q.dtype, nk, 2 * ref.UNIT[Q.dtype])
        a, b = a + nq, b + nk
    return out


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("H,Hkv,d", [(1, 1, 64), (4, 2, 128), (6, 2, 8), (5, 1, 40), (8, 1, 96), (14, 2, 72), (12, 4, 64), (16, 1, 80), (3, 3, 120), (128, 1, 32)])
def test_lengths_heads_and_sizes(H, Hkv, d, dtype):
    q = [1, 0, 130, 17, 0, 257, 64]
    _check(*_inputs(q, q, H, Hkv, d, dtype, fused=True), q, q)


@pytest.mark.parametrize("q,k", [([1], [1]), ([1], [129]), ([3], [500]), ([200], [328]), ([128, 128], [128, 256]), ([5, 40, 1], [0, 300, 1]), ([300], [40]), ([140, 2], [12, 0]), ([0, 0], [7, 0])])
@pytest.mark.parametrize("H,Hkv,d", [(2, 1, 64), (4, 4, 128), (14, 2, 128)])
def test_keys_ahead_and_rows_without_keys(q, k, H, Hkv, d):
    _check(*_inputs(q, k, H, Hkv, d, BF, 1), q, k)


@pytest.mark.parametrize("n", [127, 128, 129, 255, 256, 384, 900])
@pytest.mark.parametrize("d", [64, 128])
def test_tile_edges(n, d):
    _check(*_inputs([n, 1], [n, 1], 2, 2, d, HF, n), [n, 1], [n, 1])


def test_more_sequences_than_a_launch_takes():
    q = [(7 * i) % 5 for i in range(1300)]
    _check(*_inputs(q, q, 2, 1, 64, BF, 3), q, q)


def test_scale_and_large_scores():
    """Scores that grow along the keys, so that maxima are raised late; and a scale of the caller's."""
    q = [200]
    Q, K, V = _inputs(q, q, 2, 1, 128, BF, 4)
    K = (K * torch.linspace(0.1, 3, 200, device="cuda")[:, None, None]).to(BF)
    _check(Q, K, V, q, q, scale=0.7)
    _check(Q, K, V, q, q, scale=1e-3)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (8, 1)])
def test_what_a_row_does_not_see(dtype, d, H, Hkv):
    """NaN and infinities in other sequences, in rows that belong to none, and in later tokens leave a row's output alone; a row that sees one has it."""
    q = [100, 60, 150]
    rows = 5 + sum(q) + 40
    g = torch.Generator(device="cuda").manual_seed(5)
    Q, K, V = (torch.empty(rows, h, d, device="cuda").normal_(generator=g).to(dtype) for h in (H, Hkv, Hkv))
    starts = ref.starts(q) + 5
    plain = psa.psa_prompt_attention(Q, K, V, starts, out=torch.zeros(rows, H * d, dtype=dtype, device="cuda"))
    K2, V2 = K.clone(), V.clone()
    for t in (K2, V2):
        t[:5], t[5 + sum(q):] = float("nan"), float("inf")
        t[105:165] = float("nan")                       # the middle sequence
        t[5 + 160 + 120] = float("inf")                 # a token of the last one
    V2[5 + 160 + 140, :, 3] = float("-inf")
    lse = torch.zeros(rows, H, device="cuda")
    out = torch.full((rows, H * d), 7.0, dtype=dtype, device="cuda")
    psa.psa_prompt_attention(Q, K2, V2, starts, out=out, lse=lse)
    assert psa.psa_last_issued()[0] == psa.OK
    assert (out[:5] == 7).all() and (out[5 + sum(q):] == 7).all()
    keep = list(range(5, 105)) + list(range(165, 165 + 120))
    assert torch.equal(out[keep], plain[keep])
    assert torch.isnan(out[105:165].view(60, H, d)).all()
    assert not torch.isfinite(out[165 + 120:165 + 150]).any()
    # V alone: the scores are finite, so the outputs are infinities of V's sign, in its column only
    V3 = V.clone()
    V3[165 + 30, :, 3] = float("-inf")
    V3[165 + 129, :, 5] = float("inf")
    V3[105 + 59, :, 0] = float("nan")
    o = psa.psa_prompt_attention(Q, K, V3, starts, out=torch.zeros(rows, H * d, dtype=dtype, device="cuda")).view(rows, H, d)
    p = plain.view(rows, H, d)
    assert (o[195:315, :, 3] == float("-inf")).all() and (o[294:315, :, 5] == float("inf")).all() and torch.isnan(o[164, :, 0]).all()
    same = torch.ones(rows, H, d, dtype=torch.bool, device="cuda")
    same[195:315, :, 3] = same[294:315, :, 5] = same[164, :, 0] = False
    assert torch.equal(o[same], p[same])


def test_strides_and_given_outputs():
    q = [70, 33]
    buf = torch.empty(sum(q), 1000, device="cuda").normal_().clamp(-4, 4).to(BF)
    Q, K, V = (buf[:, a:a + h * 64].view(-1, h, 64) for a, h in ((0, 4), (320, 2), (504, 2)))
    out, lse = torch.empty(sum(q), 256, dtype=BF, device="cuda"), torch.empty(sum(q), 4, device="cuda")
    assert _check(Q, K, V, q, q, out=out, lse=lse) is out


def test_another_stream_and_no_keys_tensor():
    q = [40, 300]
    Q, K, V = _inputs(q, q, 4, 1, 128, BF, 6)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    starts = ref.starts(q)
    want = psa.psa_prompt_attention(Q, K, V, starts)
    torch.cuda.synchronize()
    got = psa.psa_prompt_attention(Q, K, V, starts, stream=s)
    s.synchronize()
    assert torch.equal(want, got)
    none = torch.empty(0, 1, 128, dtype=BF, device="cuda")
    out = psa.psa_prompt_attention(Q, none, none, starts, ref.starts([0, 0]))
    assert (out == 0).all()


def test_graph_replay():
    q = [130, 9, 70]
    Q, K, V = _inputs(q, q, 4, 2, 64, HF, 7)
    starts, out = ref.starts(q), torch.empty(sum(q), 256, dtype=HF, device="cuda")
    psa.psa_prompt_attention(Q, K, V, starts, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        psa.psa_prompt_attention(Q, K, V, starts, out=out)
    for lengths in ([100, 9, 100], [0, 209, 0], q):
        starts.copy_(ref.starts(lengths))
        graph.replay()
        graph.replay()
        got = out.clone()
        assert torch.equal(got, psa.psa_prompt_attention(Q, K, V, starts))


def test_starts_that_name_no_rows():
    Q, K, V = _inputs([50], [50], 2, 1, 64, BF, 8)
    bad = torch.tensor([0, 50, 0, 50, 0, 50] * 20, dtype=torch.int32, device="cuda")      # rows counted many times over
    out = psa.psa_prompt_attention(Q, K, V, bad, out=torch.zeros(50, 128, dtype=BF, device="cuda"))
    assert psa.psa_last_issued()[0] in (psa.OK, psa.ERR_SHAPE)
    far = torch.tensor([-7, 30, 1000], dtype=torch.int32, device="cuda")                  # rows outside the tensors are not touched
    out = psa.psa_prompt_attention(Q, K, V, far)
    assert psa.psa_last_issued()[0] == psa.OK
    assert torch.equal(out, psa.psa_prompt_attention(Q, K, V, ref.starts([30, 20])))


def test_random_batches():
    r = __import__("random").Random(11)
    for i in range(12):
        q = [r.choice([0, 1, 2, 5, 17, 60, 128, 200]) for _ in range(r.randint(1, 9))]
        k = [n + r.choice([0, 0, 1, 30, 129, -min(n, 3)]) for n in q]
        Hkv, G, d = r.choice([1, 2, 3]), r.choice([1, 2, 3, 4, 6, 7, 8, 11]), 8 * r.randint(1, 16)
        if sum(q):
            _check(*_inputs(q, k, Hkv * G, Hkv, d, r.choice([BF, HF]), i), q, k)


def test_blocks_are_counted():
    """One sequence of 300 tokens, one head: row tiles of 128 with 1, 2 and 3 key blocks."""
    Q, K, V = _inputs([300], [300], 1, 1, 64, BF, 9)
    psa.psa_prompt_attention(Q, K, V, ref.starts([300]))
    st, c = psa.psa_last_issued()
    assert st == psa.OK and c["qk_macs"] == c["pv_macs"] == 6 * 128 * 128 * 64 and c["useful_qk_macs"] == 0


def test_longer_than_one_piece():
    n = 3001
    Q, K, V = _inputs([n], [n], 2, 1, 64, BF, 10)
    starts = ref.starts([n])
    out = psa.psa_prompt_attention(Q, K, V, starts)
    rows = [0, 1, 127, 128, 1500, 2900, 3000]
    for i in rows:
        r = ref.attend(Q[i:i + 1], K[:i + 1], V[:i + 1], 1 / 8)
        ref.close(out[i:i + 1], None, r, BF, n, 2 * ref.UNIT[BF])
    assert math.isfinite(float(out.float().sum()))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("q,k,H,Hkv,d", [([3], [5000], 8, 1, 64), ([70, 1, 0], [3000, 1500, 900], 4, 2, 128), ([200], [2400], 1, 1, 80), ([5, 5, 5], [1025, 4000, 2], 12, 4, 128), ([260], [2200], 2, 2, 64),
                                         ([1], [9000], 32, 8, 128), ([1500], [1400], 2, 1, 64)])
def test_keys_in_parts(q, k, H, Hkv, d, dtype):
    """Few rows and many keys: the key blocks are shared out among CTAs.  The result does not depend on who joins the parts."""
    Q, K, V = _inputs(q, k, H, Hkv, d, dtype, 12)
    want = _check(Q, K, V, q, k)
    for _ in range(3):
        assert torch.equal(want, psa.psa_prompt_attention(Q, K, V, ref.starts(q), ref.starts(k)))
    K2, V2 = K.clone(), V.clone()
    K2[k[0] - 1], V2[k[0] - 1] = float("nan"), float("nan")         # the last token of the first sequence: its last row sees it, nobody else
    got = psa.psa_prompt_attention(Q, K2, V2, ref.starts(q), ref.starts(k))
    same = [i for i in range(sum(q)) if i != q[0] - 1]
    assert torch.equal(got[same], want[same]) and torch.isnan(got[q[0] - 1]).all()
    V2.copy_(V)
    V2[k[0] // 2, :, 1] = float("inf")
    got = psa.psa_prompt_attention(Q, K, V2, ref.starts(q), ref.starts(k)).view(-1, H, d)
    sees = [i for i in range(q[0]) if i + k[0] - q[0] >= k[0] // 2]
    assert (got[sees, :, 1] == float("inf")).all()
    got[sees, :, 1] = want.view(-1, H, d)[sees, :, 1]
    assert torch.equal(got.view(-1, H * d), want)


@pytest.mark.parametrize("q,k", [([300], [300]), ([64], [3000]), ([33, 1, 64], [900, 700, 40]), ([130, 0, 5], [2000, 50, 1]), ([520, 260], [520, 300])])
@pytest.mark.parametrize("H,Hkv,d,dtype", [(4, 2, 64, BF), (8, 2, 128, HF), (6, 2, 96, BF)])
def test_few_tiles_and_many_keys(q, k, H, Hkv, d, dtype):
    """One row tile a CTA or two, whole or in parts, by how much there is to do."""
    _check(*_inputs(q, k, H, Hkv, d, dtype, 9), q, k)
    _check(*_inputs(q * 3, k * 3, H, Hkv, d, dtype, 10), q * 3, k * 3)
