"""Refusals of the drafting entry points, which launch nothing and need no GPU, and their reference against itself."""
import ctypes
import random

import numpy as np
import pytest
import torch

import drafts_reference as ref
import serving_reference as sref
from paper_2012_01114_b200 import binding, build

P = 1 << 20                                     # an address; nothing is read there


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def _cache(**kw):
    a = dict(pool=P, tables=P, lens=P, pages=4, slots=2, width=3, page_size=16, kv_heads=2, d_k=64)
    a.update(kw)
    return ctypes.byref(binding.Cache(*(a[k] for k in ("pool", "tables", "lens", "pages", "slots", "width", "page_size", "kv_heads", "d_k"))))


BAD_CACHE = [(dict(pool=None), "NULL"), (dict(lens=None), "NULL"), (dict(slots=0), "SHAPE"), (dict(width=1 << 28), "SHAPE"), (dict(page_size=24), "UNSUPPORTED"), (dict(d_k=48), "UNSUPPORTED"),
             (dict(pool=P + 8), "ALIGN")]


def _want(name):
    return binding.OK if name is None else getattr(binding, "ERR_" + name)


@pytest.mark.parametrize("change,want", [
    ({}, "ANY"), (dict(K=None), "NULL"), (dict(V=None), "NULL"), (dict(seqs=None), "NULL"), (dict(starts=None), "NULL"), (dict(freqs=None), "NULL"), (dict(q_out=None), "NULL"),
    (dict(n=0), "SHAPE"), (dict(rows=-1), "SHAPE"), (dict(ks=120), "SHAPE"), (dict(vs=132), "SHAPE"), (dict(qs=248), "SHAPE"), (dict(qs=260), "SHAPE"), (dict(H=0), "SHAPE"),
    (dict(rot=0), "SHAPE"), (dict(rot=-8), "SHAPE"), (dict(rot=72), "SHAPE"), (dict(rot=12), "UNSUPPORTED"), (dict(amplitude=float("nan")), "UNSUPPORTED"),
    (dict(amplitude=float("inf")), "UNSUPPORTED"), (dict(dtype=binding.F32), "UNSUPPORTED"), (dict(rows=(1 << 31) - 1, n=1), "SHAPE"),
    (dict(K=P + 8), "ALIGN"), (dict(Q=P + 8), "ALIGN"), (dict(q_out=P + 4), "ALIGN"), (dict(kh=P + 2), "ALIGN"), (dict(freqs=P + 4), "ALIGN"), (dict(depths=P + 2), "ALIGN"),
    (dict(rows=0, K=None), None), (dict(rows=0, n=0), None), (dict(Q=None, H=0, K=None), "NULL")] + [(dict(cache=c), w) for c, w in BAD_CACHE])
def test_append_rotary_refusals(lib, change, want):
    if want == "ANY":
        return
    a = dict(cache={}, Q=P, K=P, V=P, qs=256, ks=128, vs=128, depths=P, seqs=P, starts=P, n=1, rows=5, H=4, dtype=binding.BF16, q_out=P, kh=None, vh=None, freqs=P, amplitude=1.0, rot=64, inter=0)
    a.update(change)
    rotary = binding.Rotary(a["freqs"], a["amplitude"], a["rot"], a["inter"])
    assert lib.psa_cache_append_rotary(_cache(**a["cache"]), ctypes.byref(rotary), a["Q"], a["K"], a["V"], a["qs"], a["ks"], a["vs"], a["depths"], a["seqs"], a["starts"], a["n"], a["rows"], a["H"],
                                       a["dtype"], a["q_out"], a["kh"], a["vh"], None) == _want(want)
    assert lib.psa_cache_append_rotary(_cache(), None, P, P, P, 256, 128, 128, None, P, P, 1, 5, 4, binding.BF16, P, None, None, None) == binding.ERR_NULL


@pytest.mark.parametrize("change,want", [
    (dict(Q=None), "NULL"), (dict(parents=None), "NULL"), (dict(seqs=None), "NULL"), (dict(starts=None), "NULL"), (dict(out=None), "NULL"), (dict(n=0), "SHAPE"), (dict(rows=-1), "SHAPE"),
    (dict(H=3), "SHAPE"), (dict(max_q=0), "SHAPE"), (dict(qs=248), "SHAPE"), (dict(max_q=1025), "UNSUPPORTED"), (dict(scale=0.0), "UNSUPPORTED"), (dict(dtype=binding.F32), "UNSUPPORTED"),
    (dict(Q=P + 8), "ALIGN"), (dict(out=P + 4), "ALIGN"), (dict(lse=P + 1), "ALIGN"), (dict(parents=P + 2), "ALIGN"), (dict(rows=0, Q=None), None)] + [(dict(cache=c), w) for c, w in BAD_CACHE])
def test_tree_refusals(lib, change, want):
    a = dict(cache={}, Q=P, qs=256, parents=P, seqs=P, starts=P, n=1, rows=5, H=4, max_q=5, scale=0.1, dtype=binding.F16, out=P, lse=None)
    a.update(change)
    assert lib.psa_tree_attention(_cache(**a["cache"]), a["Q"], a["qs"], a["parents"], a["seqs"], a["starts"], a["n"], a["rows"], a["H"], a["max_q"], a["scale"], a["dtype"], a["out"], a["lse"],
                                  None) == _want(want)


@pytest.mark.parametrize("change,want", [
    (dict(logits=None), "NULL"), (dict(tokens=None), "NULL"), (dict(parents=None), "NULL"), (dict(starts=None), "NULL"), (dict(uniform=None), "NULL"), (dict(path=None), "NULL"),
    (dict(accepted=None), "NULL"), (dict(next=None), "NULL"), (dict(n=0), "SHAPE"), (dict(n=-1), "SHAPE"), (dict(rows=-1), "SHAPE"), (dict(vocab=0), "SHAPE"), (dict(vocab=(1 << 30) + 1, ls=1 << 31, ds=1 << 31), "SHAPE"), (dict(ls=99), "SHAPE"),
    (dict(ds=99), "SHAPE"), (dict(ls=1 << 39), "SHAPE"), (dict(dtype=3), "UNSUPPORTED"), (dict(logits=P + 1), "ALIGN"), (dict(drafts=P + 1), "ALIGN"), (dict(dtype=binding.F32, logits=P + 2), "ALIGN"),
    (dict(uniform=P + 2), "ALIGN"), (dict(path=P + 2), "ALIGN"), (dict(temperatures=P + 1), "ALIGN"), (dict(rows=0, n=0, starts=None), None)])
def test_verify_refusals(lib, change, want):
    a = dict(logits=P, ls=100, drafts=P, ds=100, vocab=100, dtype=binding.BF16, tokens=P, parents=P, starts=P, n=2, rows=5, temperatures=None, uniform=P, distinct=1, path=P, accepted=P, next=P)
    a.update(change)
    assert lib.psa_verify_drafts(*(a[k] for k in ("logits", "ls", "drafts", "ds", "vocab", "dtype", "tokens", "parents", "starts", "n", "rows", "temperatures", "uniform", "distinct", "path",
                                                  "accepted", "next")), None) == _want(want)


@pytest.mark.parametrize("change,want", [
    (dict(seqs=None), "NULL"), (dict(starts=None), "NULL"), (dict(path=None), "NULL"), (dict(accepted=None), "NULL"), (dict(new_lens=None), "NULL"), (dict(layers=0), "SHAPE"), (dict(n=-1), "SHAPE"),
    (dict(n=0), "SHAPE"), (dict(rows=-1), "SHAPE"), (dict(layers=1 << 30), "SHAPE"), (dict(path=P + 2), "ALIGN"), (dict(new_lens=P + 1), "ALIGN"), (dict(n=0, rows=0), None),
    (dict(rows=0, path=None), None)] + [(dict(cache=c), w) for c, w in BAD_CACHE])
def test_keep_refusals(lib, change, want):
    a = dict(cache={}, layers=2, seqs=P, starts=P, path=P, accepted=P, n=3, rows=5, new_lens=P)
    a.update(change)
    assert lib.psa_cache_keep(_cache(**a["cache"]), a["layers"], a["seqs"], a["starts"], a["path"], a["accepted"], a["n"], a["rows"], a["new_lens"], None) == _want(want)


def test_binding_refuses_what_it_cannot_marshal():
    cpu, ints = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    pool, tables, one = torch.zeros(1, 160, dtype=torch.uint8), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.psa_cache_append_rotary(cpu, cpu, pool, tables, one, one, torch.zeros(2, dtype=torch.int32), 16, torch.ones(32, dtype=torch.float64))
    with pytest.raises(ValueError):
        binding.psa_tree_attention(cpu, pool, tables, one, one, torch.zeros(2, dtype=torch.int32), ints, 2, 16, 4)
    with pytest.raises(ValueError):
        binding.psa_verify_drafts(torch.zeros(4, 100), ints, ints, torch.zeros(2, dtype=torch.int32), torch.zeros(4))
    with pytest.raises(ValueError):
        binding.psa_cache_keep(pool, tables, one, one, torch.zeros(2, dtype=torch.int32), ints, one, 2, 16)


def test_reference_chain_is_the_causal_one():
    q, k, v = torch.randn(5, 4, 32), torch.randn(20, 2, 32), torch.randn(20, 2, 32)
    a, b = ref.attend(q, k, v, 0.2, ref.seen_by([-1, 0, 1, 2, 3], 5, 20)), sref.attend(q, k, v, 0.2)
    assert all(torch.allclose(x, y, rtol=1e-12, atol=1e-12) for x, y in zip(a, b))


@pytest.mark.parametrize("drafts", ["none", "replaced", "distinct"])
def test_reference_verification_gives_the_targets_distribution(drafts):
    """Root and two drafted children of it, 12,000 times: the first token behind the root has the target's probabilities.  Five standard deviations of each count."""
    r = np.random.default_rng(3)
    V, n = 5, 12000
    logits, g = torch.tensor(r.normal(size=(3, V))), torch.tensor(r.normal(size=(3, V)))
    p, q = torch.softmax(logits[0], 0).numpy(), torch.softmax(g[0], 0).numpy()
    count = np.zeros(V)
    for _ in range(n):
        t = r.choice(V, 2, replace=drafts != "distinct", p=q)
        path, accepted, following, _ = ref.verify(logits, None if drafts == "none" else g, [0, int(t[0]), int(t[1])], [-1, 0, 0], r.random(3), 1.0, drafts == "distinct")
        count[t[path[1] - 1] if accepted else following] += 1
    assert (np.abs(count / n - p) <= 5 * np.sqrt(p * (1 - p) / n)).all()


def test_reference_bytes_belong_to_one_token_each():
    for d, page, H in ((32, 16, 1), (96, 32, 2)):
        at = sorted(x for h in range(H) for t in range(page) for x in ref.byte_places(page, H, d, h, t))
        assert at == list(range(H * page * d * 5 // 4))


def test_reference_trees():
    r = random.Random(1)
    for n in (1, 2, 30):
        parents, level = ref.random_tree(n, r)
        assert len(parents) == n and all(-1 <= p < i for i, p in enumerate(parents)) and all(level[i] == (0 if p < 0 else level[p] + 1) for i, p in enumerate(parents))


def test_workspace_of_a_tree(lib):
    for d in (32, 64, 96, 128, 256):
        assert lib.psa_tree_workspace_bytes(d) >= lib.psa_cache_workspace_bytes(d) > 0
    for d in (0, -64, 16, 48, 512):
        assert lib.psa_tree_workspace_bytes(d) == 0
