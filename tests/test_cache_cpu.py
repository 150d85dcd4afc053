"""Paged HIF4 cache without a GPU: size queries, refusals, and the tests' own restatement of the page format."""
import ctypes as C

import numpy as np
import pytest

from oracle import hifa4_oracle as orc
from tests import cache_reference as ref


@pytest.fixture(scope="module")
def hb():
    from paper_2607_04302_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _cache(hb, **over):
    f = dict(Hkv=8, d=128, in_dtype=hb.BF16, n_pages=10, pages=256, n_tails=2, v_tail=256)
    f.update(over)
    return hb._Cache(*[f[n] for n, _ in hb._Cache._fields_])


def _seqs(hb, **over):
    f = dict(B=2, max_pages=5, block_table=256, kv_lens=256, tail_slots=None)
    f.update(over)
    return hb._Seqs(*[f[n] for n, _ in hb._Seqs._fields_])


def _query(hb, **over):
    f = dict(Hq=32, q_to_kv=None, N=1, causal=0, out_dtype=hb.BF16, softmax_scale=0.0)
    f.update(over)
    return hb._CacheQuery(*[f[n] for n, _ in hb._CacheQuery._fields_])


def test_sizes(hb):
    assert [hb.cache_page_bytes(d) for d in (64, 128, 256, 96, 0, -64)] == [4736, 9472, 18944, 0, 0, 0]
    size = hb.lib().hifa4_cache_decode_workspace_bytes
    q = _query(hb)
    small = size(C.byref(_cache(hb)), 2, 5, C.byref(q), 0)
    assert small > 0 and size(C.byref(_cache(hb)), 2, 5, C.byref(q), 1) > small
    assert size(C.byref(_cache(hb, d=96)), 2, 5, C.byref(q), 0) == 0
    assert size(C.byref(_cache(hb)), 0, 5, C.byref(q), 0) == 0
    assert size(C.byref(_cache(hb)), 2, 5, C.byref(_query(hb, N=2)), 0) == 0
    assert size(C.byref(_cache(hb)), 2, 5, C.byref(_query(hb, Hq=30)), 0) == 0
    assert hb.lib().hifa4_cache_attention_workspace_bytes(C.byref(_cache(hb)), 2, 5, C.byref(_query(hb, N=100))) > 0


CACHES = [(dict(pages=None), 1), (dict(pages=264), 1), (dict(Hkv=0), 1), (dict(Hkv=257), 1), (dict(n_pages=0), 1), (dict(in_dtype=2), 1),
          (dict(d=96), 2)]
SEQS = [(dict(B=0), 1), (dict(max_pages=0), 1), (dict(block_table=None), 1), (dict(kv_lens=None), 1), (dict(B=10000), 2)]


def _p(x):
    return C.byref(x)


@pytest.mark.parametrize("cache,seqs,want", [(c, {}, r) for c, r in CACHES + [(dict(v_tail=None), 1), (dict(v_tail=8), 1), (dict(n_tails=0), 1)]] +
                         [({}, s, r) for s, r in SEQS])
def test_append_refuses(hb, cache, seqs, want):
    f = hb.lib().hifa4_cache_append
    assert f(_p(_cache(hb, **cache)), _p(_seqs(hb, **seqs)), 1, None, 256, None, 256, None, None, None, None) == want


def test_append_and_read_refuse_tensors(hb):
    c, s = _cache(hb), _seqs(hb)
    f = hb.lib().hifa4_cache_append
    bad, good = hb._Strides(1024, 12, 128), hb._Strides(1024, 128, 128)
    for n, k, ks, v, vs in ((0, 256, None, 256, None), (1, None, None, 256, None), (1, 256, None, None, None), (1, 258, None, 256, None),
                            (1, 256, bad, 256, good), (1, 256, good, 256, bad)):
        assert f(_p(c), _p(s), n, None, k, ks and _p(ks), v, vs and _p(vs), None, None, None) == 1
    r = hb.lib().hifa4_cache_read
    assert r(_p(c), _p(s), 0, None, hb.BF16, 256, 256, None, None) == 1
    assert r(_p(c), _p(s), 1, None, hb.BF16, None, 256, None, None) == 1
    assert r(_p(c), _p(s), 1, None, 5, 256, 256, None, None) == 1
    assert r(_p(c), _p(s), 1, None, hb.F16, 256, 256, None, None) == 2
    assert r(None, _p(s), 1, None, hb.BF16, 256, 256, None, None) == 1


@pytest.mark.parametrize("cache,seqs,query,want", [(c, {}, {}, r) for c, r in CACHES] + [({}, s, {}, r) for s, r in SEQS] + [
    ({}, {}, dict(Hq=30), 1), ({}, {}, dict(Hq=0), 1), ({}, {}, dict(N=0), 1), ({}, {}, dict(out_dtype=3), 1), ({}, {}, dict(causal=2), 1),
    ({}, {}, dict(softmax_scale=-1.0), 1), ({}, {}, dict(softmax_scale=float("inf")), 1)])
def test_attention_refuses(hb, cache, seqs, query, want):
    big = 1 << 40
    args = [256, None, None, 256]
    f, g = hb.lib().hifa4_cache_decode, hb.lib().hifa4_cache_attention
    c, s, q = _cache(hb, **cache), _seqs(hb, **seqs), _query(hb, **query)
    assert f(_p(c), _p(s), _p(q), *args, None, None, None, 256, big, None, None) == want
    assert g(_p(c), _p(s), _p(q), *args, 256, big, None, None) == want


def test_attention_refuses_tensors_and_workspaces(hb):
    f = hb.lib().hifa4_cache_decode
    c, s, q = _cache(hb), _seqs(hb), _query(hb)
    need = hb.lib().hifa4_cache_decode_workspace_bytes(_p(c), 2, 5, _p(q), 0)
    bad = hb._Strides(4096, 4, 0)

    def call(qp=256, st=None, out=256, w=None, w_out=None, ws=256, nb=need, query=q):
        return f(_p(c), _p(s), _p(query), qp, st and _p(st), None, out, None, w, w_out, ws, nb, None, None)

    assert call(qp=None) == call(qp=260) == call(st=bad) == call(out=None) == call(w=256) == 1
    assert call(ws=None) == call(nb=need - 1) == call(ws=128) == call(w_out=256) == 3
    assert call(query=_query(hb, N=2)) == 1
    wrong = (C.c_int * 32)(*([0] * 31 + [8]))
    assert call(query=_query(hb, q_to_kv=C.cast(wrong, C.POINTER(C.c_int)))) == 1
    import torch
    if not torch.cuda.is_available():
        assert call() in (4, 5)                          # a well-formed call is refused for want of a device, never run on the CPU


def test_refuses_what_wide_loads_and_stores_cannot_take(hb):
    """Factors are read and the cache's values stored 16 bytes at a time."""
    c, s, q = _cache(hb), _seqs(hb), _query(hb)
    for off, want in ((0, (4, 5)), (4, (1,)), (8, (1,))):
        got = [hb.lib().hifa4_cache_read(_p(c), _p(s), 1, None, hb.BF16, 256 + off, 256, None, None),
               hb.lib().hifa4_cache_read(_p(c), _p(s), 1, None, hb.F32, 256, 256 + off, None, None),
               hb.lib().hifa4_cache_append(_p(c), _p(s), 1, None, 256, None, 256, None, 256 + off, None, None),
               hb.lib().hifa4_cache_decode(_p(c), _p(s), _p(q), 256, None, 256 + off, 256, None, None, None, 256, 1 << 40, None, None),
               hb.lib().hifa4_cache_attention(_p(c), _p(s), _p(_query(hb, N=40)), 256, None, 256 + off, 256, 256, 1 << 40, None, None)] \
            if off or not _has_gpu() else []
        assert all(g in want for g in got), (off, got)


def test_decode_does_not_look_at_the_token_stride(hb):
    """q of one token: what the third stride holds does not matter (hifa4.h: unused)."""
    if not _has_gpu():
        st = hb._Strides(4096, 128, 3)
        assert hb.lib().hifa4_cache_decode(_p(_cache(hb)), _p(_seqs(hb)), _p(_query(hb)), 256, _p(st), None, 256, None, None, None, 256,
                                           1 << 40, None, None) in (4, 5)


def _has_gpu():
    import torch
    return torch.cuda.is_available()                     # (made-up addresses are for hosts without one)


def test_evict_refuses(hb):
    f = hb.lib().hifa4_cache_evict

    def call(seqs=None, w=256, keep=4, first=1, last=1, outs=(256,) * 5):
        return f(_p(seqs or _seqs(hb)), w, keep, first, last, *outs, None, None)

    assert call(w=None) == call(keep=1) == call(first=-1) == call(last=0) == call(keep=-1) == 1
    assert call(first=2 ** 31 - 1, last=2 ** 31 - 1, keep=2 ** 31 - 1) == 1
    for i in range(5):
        assert call(outs=tuple(None if j == i else 256 for j in range(5))) == 1
    for over, want in SEQS[:-1]:
        assert call(seqs=_seqs(hb, **over)) == want


@pytest.mark.parametrize("d", [64, 128, 256])
def test_page_format_restatement(oracle, d):
    """The tests' packing and unpacking agree with the oracle's values, and the codes take 4.625 bits a value."""
    rng = np.random.default_rng(d)
    k, v = rng.standard_normal((64, d)), rng.standard_normal((64, d))
    k, v = k.astype(np.float16).astype(np.float64), v.astype(np.float16).astype(np.float64)
    page = ref.page_bytes(k, v)
    assert page.size == 74 * d
    K, V = ref.values(page)
    assert np.array_equal(K, orc.hif4_quantize_rows(k)[2])
    assert np.array_equal(V.T, orc.hif4_quantize_rows(np.ascontiguousarray(v.T))[2])


def test_reference_agrees_with_the_plain_forms(oracle):
    """Two packings written apart: the benchmark's plain form against the tests'."""
    import torch
    from perf import operators as ops
    gen = torch.Generator().manual_seed(1)
    k, v = torch.randn((3, 64, 128), generator=gen).half().float(), torch.randn((3, 64, 128), generator=gen).half().float()
    pages = ops._pack(k, v)
    for i in range(3):
        assert np.array_equal(pages[i].numpy(), ref.page_bytes(k[i].double().numpy(), v[i].double().numpy()))
    K, V = ops._unpack(pages)
    assert np.array_equal(K[1].double().numpy(), ref.values(pages[1].numpy())[0])
    assert np.array_equal(V[1].double().numpy(), ref.values(pages[1].numpy())[1])
