"""The serving entry points' refusals, which launch nothing and need no GPU, and the reference layout of the cache against itself."""
import ctypes

import pytest
import torch

import serving_reference as ref
from paper_2012_01114_b200 import binding, build

P = 1 << 20                                     # an address; nothing is read there


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def _prompt(lib, Q=P, K=P, V=P, qs=512, ks=256, vs=256, q_starts=P, k_starts=P, n=2, q_rows=10, k_rows=10, H=4, Hkv=2, d=128, scale=0.1, dtype=binding.BF16, out=P, lse=None):
    return lib.psa_prompt_attention(Q, K, V, qs, ks, vs, q_starts, k_starts, n, q_rows, k_rows, H, Hkv, d, scale, dtype, out, lse, None)


@pytest.mark.parametrize("change,want", [
    (dict(Q=None), "NULL"), (dict(K=None), "NULL"), (dict(V=None), "NULL"), (dict(out=None), "NULL"), (dict(q_starts=None), "NULL"),
    (dict(n=0), "SHAPE"), (dict(q_rows=-1), "SHAPE"), (dict(k_rows=-1), "SHAPE"), (dict(H=5), "SHAPE"), (dict(H=0), "SHAPE"), (dict(Hkv=0), "SHAPE"), (dict(d=0), "SHAPE"),
    (dict(qs=504), "SHAPE"), (dict(qs=516), "SHAPE"), (dict(ks=248), "SHAPE"), (dict(vs=257), "SHAPE"), (dict(k_starts=None, k_rows=11), "SHAPE"),
    (dict(d=136, qs=1024, ks=512, vs=512), "UNSUPPORTED"), (dict(d=12), "UNSUPPORTED"), (dict(dtype=binding.F32), "UNSUPPORTED"), (dict(dtype=7), "UNSUPPORTED"),
    (dict(H=258, d=8, qs=4096), "UNSUPPORTED"), (dict(scale=0.0), "UNSUPPORTED"), (dict(scale=-1.0), "UNSUPPORTED"), (dict(scale=float("nan")), "UNSUPPORTED"), (dict(scale=float("inf")), "UNSUPPORTED"),
    (dict(Q=P + 8), "ALIGN"), (dict(K=P + 2), "ALIGN"), (dict(V=P + 8), "ALIGN"), (dict(out=P + 8), "ALIGN"), (dict(lse=P + 2), "ALIGN"), (dict(q_starts=P + 1), "ALIGN"),
    (dict(q_rows=0, Q=None), None)])
def test_prompt_refusals(lib, change, want):
    assert _prompt(lib, **change) == (binding.OK if want is None else getattr(binding, "ERR_" + want))


def _cache(**kw):
    a = dict(pool=P, tables=P, lens=P, pages=4, slots=2, width=3, page_size=16, kv_heads=2, d_k=64)
    a.update(kw)
    return ctypes.byref(binding.Cache(*(a[k] for k in ("pool", "tables", "lens", "pages", "slots", "width", "page_size", "kv_heads", "d_k"))))


CACHE = [(dict(pool=None), "NULL"), (dict(tables=None), "NULL"), (dict(lens=None), "NULL"), (dict(pages=0), "SHAPE"), (dict(slots=0), "SHAPE"), (dict(width=-1), "SHAPE"), (dict(page_size=0), "SHAPE"),
         (dict(kv_heads=0), "SHAPE"), (dict(width=1 << 28), "SHAPE"), (dict(page_size=24), "UNSUPPORTED"), (dict(d_k=48), "UNSUPPORTED"), (dict(d_k=160), "UNSUPPORTED"), (dict(pool=P + 8), "ALIGN"),
         (dict(tables=P + 1), "ALIGN")]


@pytest.mark.parametrize("change,want", CACHE)
def test_cache_refusals(lib, change, want):
    want = getattr(binding, "ERR_" + want)
    assert lib.psa_cache_append(_cache(**change), P, P, 128, 128, P, P, 1, 5, binding.BF16, None, None, None) == want
    assert lib.psa_cache_attention(_cache(**change), P, 256, P, P, 1, 5, 4, 1, 0.1, binding.BF16, P, None, None) == want


def test_append_and_attention_refusals(lib):
    def append(K=P, V=P, ks=128, vs=128, seqs=P, starts=P, n=1, rows=5, dtype=binding.F16, kh=None, vh=None):
        return lib.psa_cache_append(_cache(), K, V, ks, vs, seqs, starts, n, rows, dtype, kh, vh, None)

    def attend(Q=P, qs=256, seqs=P, starts=P, n=1, rows=5, H=4, max_q=1, scale=0.1, dtype=binding.F16, out=P, lse=None):
        return lib.psa_cache_attention(_cache(), Q, qs, seqs, starts, n, rows, H, max_q, scale, dtype, out, lse, None)

    for kw in (dict(K=None), dict(V=None), dict(seqs=None), dict(starts=None)):
        assert append(**kw) == binding.ERR_NULL
    for kw in (dict(n=0), dict(rows=-1), dict(ks=120), dict(vs=132)):
        assert append(**kw) == binding.ERR_SHAPE
    for kw in (dict(K=P + 8), dict(kh=P + 2), dict(vh=P + 8), dict(starts=P + 2)):
        assert append(**kw) == binding.ERR_ALIGN
    assert append(dtype=binding.F32) == binding.ERR_UNSUPPORTED and append(rows=0, K=None) == binding.OK
    for kw in (dict(Q=None), dict(seqs=None), dict(starts=None), dict(out=None)):
        assert attend(**kw) == binding.ERR_NULL
    for kw in (dict(n=0), dict(rows=-1), dict(H=3), dict(H=0), dict(max_q=0), dict(qs=248), dict(qs=260)):
        assert attend(**kw) == binding.ERR_SHAPE
    for kw in (dict(Q=P + 8), dict(out=P + 4), dict(lse=P + 1)):
        assert attend(**kw) == binding.ERR_ALIGN
    for kw in (dict(dtype=binding.F32), dict(scale=0.0), dict(scale=float("nan"))):
        assert attend(**kw) == binding.ERR_UNSUPPORTED
    assert attend(rows=0, Q=None) == binding.OK
    assert lib.psa_cache_append(None, P, P, 128, 128, P, P, 1, 5, binding.BF16, None, None, None) == binding.ERR_NULL


def test_page_refusals(lib):
    def pages(**kw):
        a = dict(tables=P, lens=P, refs=P, slots=2, width=3, pages=4, page_size=16)
        a.update(kw)
        return ctypes.byref(binding.Pages(*(a[k] for k in ("tables", "lens", "refs", "slots", "width", "pages", "page_size"))))

    for kw, want in ((dict(tables=None), "NULL"), (dict(refs=None), "NULL"), (dict(slots=0), "SHAPE"), (dict(pages=0), "SHAPE"), (dict(page_size=0), "SHAPE"), (dict(refs=P + 2), "ALIGN")):
        want = getattr(binding, "ERR_" + want)
        assert lib.psa_pages_free(pages(**kw), P, 1, None) == want
        assert lib.psa_pages_fork(pages(**kw), P, P, 1, None) == want
        assert lib.psa_pages_reserve(pages(**kw), P, 160, 1, P, P, 1, P, None) == want
        assert lib.psa_pages_compact(pages(**kw), P, 160, 1, P, P, P, P, None) == want
    assert lib.psa_pages_free(pages(lens=None), P, 1, None) == binding.ERR_NULL
    assert lib.psa_pages_free(pages(), P, -1, None) == binding.ERR_SHAPE and lib.psa_pages_free(pages(), None, 0, None) == binding.OK
    assert lib.psa_pages_fork(pages(), P, None, 1, None) == binding.ERR_NULL
    for args, want in (((None, 160, 1, P, P, 1, P), "NULL"), ((P, 0, 1, P, P, 1, P), "SHAPE"), ((P, 160, 0, P, P, 1, P), "SHAPE"), ((P, 168, 1, P, P, 1, P), "ALIGN"), ((P + 8, 160, 1, P, P, 1, P), "ALIGN"),
                       ((P, 160, 1, P, P, 4097, P), "UNSUPPORTED"), ((P, 160, 1, P, P, 1, None), "NULL"), ((P, 160, 1, P, P, 1, P + 1), "ALIGN")):
        assert lib.psa_pages_reserve(pages(), *args, None) == getattr(binding, "ERR_" + want)
    assert lib.psa_pages_compact(pages(lens=None), P, 160, 1, None, P, P, P, None) == binding.ERR_NULL
    for args, want in (((None, 4, P, 4, 160, 1, P, P, 1), "NULL"), ((P, 0, P, 4, 160, 1, P, P, 1), "SHAPE"), ((P, 4, P, 4, 24, 1, P, P, 1), "ALIGN"), ((P, 4, P, 4, 160, 1, None, P, 1), "NULL")):
        assert lib.psa_pages_copy(*args, None) == getattr(binding, "ERR_" + want)
    assert lib.psa_pages_copy(P, 4, P, 4, 160, 1, None, None, 0, None) == binding.OK


def test_sizes(lib):
    assert binding.psa_cache_page_bytes(8, 64, 128) == 8 * 64 * 128 * 5 // 4
    assert [binding.psa_cache_page_bytes(*a) for a in ((0, 16, 64), (1, 8, 64), (1, 16, 72), (1, -16, 64))] == [0] * 4
    assert binding.psa_cache_workspace_bytes(128) > 256 and binding.psa_cache_workspace_bytes(100) == 0
    assert binding.psa_pages_workspace_bytes(1000, 10) >= 256 + 4000 and binding.psa_pages_workspace_bytes(0, 1) == 0


def test_binding_refuses_what_it_cannot_marshal():
    cpu = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.psa_prompt_attention(cpu, cpu, cpu, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        binding.psa_cache_append(cpu, cpu, torch.zeros(1, 160, dtype=torch.uint8), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                                 torch.zeros(2, dtype=torch.int32), 16)


@pytest.mark.parametrize("d", [32, 96, 128])
def test_reference_layouts_agree(d):
    """Token by token and block by block, every byte of a block written exactly once."""
    k, v = torch.randn(32, d), torch.randn(32, d)
    kq, vq = ref.quantise(k), ref.quantise(v)
    page = torch.zeros(40 * d, dtype=torch.uint8)
    for t in range(32):
        ref.put(page, 0, 32, d, t, [x[t] for x in kq], [x[t] for x in vq])
    assert torch.equal(page.view(2, -1), ref.block_images(kq, vq, 32))
    ones = tuple(torch.full_like(x, 15) if i == 0 else torch.full_like(x, -1).view(torch.int16).fill_(-1).view(torch.float16) for i, x in enumerate(kq))
    assert (ref.block_images(ones, ones, 32) == 255).all()
    assert ((ref.held(*kq) - k.double()).abs().unflatten(-1, (-1, 32)).amax(-1) <= kq[1].double() / 32 * 1.001 + 2.0 ** -10 * (kq[1].double() + kq[2].double().abs())).all()


def test_empty_batches_are_no_error(lib):
    assert _prompt(lib, n=0, q_rows=0) == binding.OK
    assert lib.psa_cache_append(_cache(), None, None, 128, 128, None, None, 0, 0, binding.BF16, None, None, None) == binding.OK
    assert lib.psa_cache_attention(_cache(), None, 256, None, None, 0, 0, 4, 1, 0.1, binding.BF16, None, None, None) == binding.OK
