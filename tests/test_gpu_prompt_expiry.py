"""Calls of psa_prompt_attention behind one whose waits ran out.  Such a call leaves arrival counts of rows in parts that are not zero; the library's self-test leaves the same
(nothing is broken on purpose, and no production kernel's wait runs out here).  Nobody asks for the status in between."""
import pytest
import torch

import serving_reference as ref
from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu
SHAPES = [([3], [5000], 8, 1, 64, torch.bfloat16), ([70, 1, 0], [3000, 1500, 900], 4, 2, 128, torch.float16), ([5, 5, 5], [1025, 4000, 2], 12, 4, 128, torch.bfloat16)]


class Call:
    def __init__(self, q, k, H, Hkv, d, dtype):
        g = torch.Generator(device="cuda").manual_seed(17)
        self.Q, self.K, self.V = (torch.empty(s, device="cuda").normal_(generator=g).clamp(-4, 4).to(dtype) for s in ((sum(q), H, d), (sum(k), Hkv, d), (sum(k), Hkv, d)))
        self.q, self.k, self.qs, self.ks, self.dtype = q, k, ref.starts(q), ref.starts(k), dtype
        assert psa.psa_prompt_workspace_bytes(len(q), sum(q), sum(k), H, Hkv, d) > 256                    # (key blocks are cut into parts)

    def run(self, out=None):
        self.lse = torch.full(self.Q.shape[:2], float("nan"), device="cuda")
        return psa.psa_prompt_attention(self.Q, self.K, self.V, self.qs, self.ks, lse=self.lse, out=out)

    def right(self, out, lse=True):
        a = b = 0
        for nq, nk in zip(self.q, self.k):
            if nq:
                r = ref.attend(self.Q[a:a + nq], self.K[b:b + nk], self.V[b:b + nk], self.Q.shape[2] ** -0.5)
                ref.close(out[a:a + nq], self.lse[a:a + nq] if lse else None, r, self.dtype, nk, 2 * ref.UNIT[self.dtype])
            a, b = a + nq, b + nk


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_calls_behind_an_expired_one(shape):
    c, other = Call(*SHAPES[shape]), Call(*SHAPES[shape - 1])
    want, want_other = c.run(), other.run()
    for between in (lambda: None, lambda: psa.psa_pages_copy(*(torch.zeros(1, 16, dtype=torch.uint8, device="cuda"),) * 2, *(torch.zeros(1, dtype=torch.int32, device="cuda"),) * 2)):
        psa.psa_selftest_wait_expiry(limit_us=1000)
        between()
        out = c.run()
        assert psa.psa_last_issued()[0] == psa.OK
        c.right(out)
        for _ in range(3):                       # and in parts again, as before
            assert torch.equal(c.run(), want) and torch.equal(other.run(), want_other)
        psa.psa_selftest_wait_expiry(limit_us=1000)
        psa.psa_selftest_wait_expiry(limit_us=1000)
        other.right(other.run())
        assert torch.equal(c.run(), want)


def test_replays_behind_an_expired_call():
    c, other = Call(*SHAPES[0]), Call(*SHAPES[1])
    want, want_other = c.run(), other.run()
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(out)
    graph.replay()
    assert torch.equal(out, want)
    psa.psa_selftest_wait_expiry(limit_us=1000)
    for _ in range(3):                           # no other call comes: without parts
        out.fill_(7)
        graph.replay()
        c.right(out, lse=False)
    assert torch.equal(other.run(), want_other)
    for _ in range(2):
        out.fill_(7)
        graph.replay()
        assert torch.equal(out, want)
