"""Calls of the paged HIF4 cache that its documentation allows, or that the binding has to refuse, beside those of test_gpu_cache.py."""
import math

import pytest
import torch

from tests import cache_reference as ref
from tests.test_gpu_cache import DEV, DT, P_BITS, check_attention, hb, ints, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_read_without_tensors_of_the_caller(dtype):
    """Rows at or behind a sequence's end hold zeros, not what the memory held before."""
    lens, H, d, n = [70, 0, 130], 2, 64, 200
    cache, table, k, v, s, inv_s = make_cache(lens, H, d, "fp16")
    old = [torch.full((3, H, n, d), math.nan, dtype=dtype, device=DEV) for _ in range(2)]
    del old                                                  # the allocator gives the same memory out again
    got = hb().cache_read(cache, table, ints(lens), n, start=ints([3, 0, 0]), out_dtype={torch.bfloat16: hb().BF16, torch.float32: hb().F32}[dtype])
    for b, (x, at) in enumerate(zip(lens, (3, 0, 0))):
        for h in range(H):
            for out, want in zip(got, ref.sequence(cache.pages.cpu(), table[b].cpu(), x, h)):
                m = max(x - at, 0)
                assert torch.equal(out[b, h, :m].double().cpu(), want[at:]) and (out[b, h, m:] == 0).all()


def test_outputs_over_the_queries_are_refused():
    cache, table, k, v, s, inv_s = make_cache([100], 2, 64, "fp16")
    q = torch.randn((1, 4, 64), device=DEV).half()
    q4 = torch.randn((1, 4, 30, 64), device=DEV).half()
    for call in (lambda: hb().cache_decode(q, cache, table, ints([100]), out=q),
                 lambda: hb().cache_attention(q4, cache, table, ints([100]), False, out=q4)):
        with pytest.raises(AssertionError):
            call()


def widened(table, width):
    return torch.cat([table, torch.full((table.shape[0], width - table.shape[1]), -1, dtype=torch.int32, device=DEV)], 1).contiguous()


@pytest.mark.parametrize("Hq,Hkv,d,N,dtype,causal", [(8, 2, 128, 40, "bf16", True), (4, 2, 64, 30, "fp16", False), (8, 2, 64, 100, "bf16", True),
                                                     (2, 1, 256, 40, "bf16", False), (8, 2, 128, 300, "bf16", True)])
def test_tables_much_wider_than_their_sequences(Hq, Hkv, d, N, dtype, causal):
    """What a captured graph of a growing batch has: entries of -1 behind the sequences' pages, which nothing reads.  Many pieces of the
    blocks are without pages."""
    lens = [300, 1, 0, 130]
    cache, table, k, v, s, inv_s = make_cache(lens, Hkv, d, dtype)
    wide, status = widened(table, 700), torch.zeros(1, dtype=torch.int32, device=DEV)
    q = (torch.randn((4, Hq, N, d), generator=torch.Generator().manual_seed(N)) * 2).to(DT[dtype])
    out = hb().cache_attention(q.to(DEV), cache, wide, ints(lens), causal, s=s, d_status=status)
    r = ref.attend(q, cache.pages.cpu(), table.cpu(), lens, s.cpu(), causal=causal)
    check_attention(out, r, d, P_BITS[dtype])
    assert (out.cpu()[r.lse == -math.inf] == 0).all()
    q1 = q[:, :, 0].contiguous().to(DEV)
    w, w_wide = torch.full(table.shape, 0.5, device=DEV), torch.full(wide.shape, 0.5, device=DEV)
    one = hb().cache_decode(q1, cache, table, ints(lens), s=s, page_weight=w, page_weight_out=w)
    again = hb().cache_decode(q1, cache, wide, ints(lens), s=s, page_weight=w_wide, page_weight_out=w_wide, d_status=status)
    assert torch.equal(one, again) and torch.equal(w, w_wide[:, :table.shape[1]]) and (w_wide[:, table.shape[1]:] == 0.5).all()
    r = hb().cache_evict(wide, ints(lens), w_wide, 2, d_status=status)
    assert r.kv_lens.tolist() == [300 - 3 * 64, 1, 0, 130 - 64] and r.n_freed.tolist() == [3, 0, 0, 1] and status.item() == 0


@pytest.mark.parametrize("Hq,Hkv,d,N,dtype", [(4, 1, 128, 30, "bf16"), (2, 2, 64, 77, "fp16"), (1, 1, 64, 128, "bf16"), (3, 3, 128, 20, "bf16")])
def test_two_tiles_on_the_same_rows_with_late_maxima(Hq, Hkv, d, N, dtype):
    """Keys grow along the sequence, so that a tile has O to rescale at its last pages; odd and even numbers of pages."""
    lens = [64 * p - x for p, x in ((1, 0), (2, 7), (3, 0), (4, 1), (5, 63), (6, 0), (7, 30), (11, 0), (12, 5))]
    B, n = len(lens), max(lens)
    gen = torch.Generator().manual_seed(N)
    grow = 0.1 + 4.0 * (torch.arange(n) // 64)[:, None] / 12
    k, v = (torch.randn((B, Hkv, n, d), generator=gen) * grow).to(DT[dtype]), torch.randn((B, Hkv, n, d), generator=gen).to(DT[dtype])
    cache = hb().alloc_cache(B * 12, Hkv, d, DT[dtype], DEV, B)
    table = torch.randperm(B * 12, generator=gen).int().view(B, 12).to(DEV).contiguous()
    hb().cache_append(cache, k.to(DEV), v.to(DEV), table, ints(lens), n_new=ints(lens))
    q = (torch.randn((B, Hq, N, d), generator=gen) * 2).to(DT[dtype])
    out = hb().cache_attention(q.to(DEV), cache, table, ints(lens), False)
    check_attention(out, ref.attend(q, cache.pages.cpu(), table.cpu(), lens), d, P_BITS[dtype])
    for _ in range(30):
        assert torch.equal(out, hb().cache_attention(q.to(DEV), cache, table, ints(lens), False))


def test_queries_shared_by_a_batch():
    """One query for all sequences, as a view with a stride of zero."""
    lens = [100, 700]
    cache, table, k, v, s, inv_s = make_cache(lens, 2, 128, "bf16")
    q = torch.randn((1, 4, 40, 128), generator=torch.Generator().manual_seed(3)).bfloat16().to(DEV)
    kv = ints(lens)
    assert torch.equal(hb().cache_attention(q.expand(2, -1, -1, -1), cache, table, kv, True, s=s),
                       hb().cache_attention(q.repeat(2, 1, 1, 1), cache, table, kv, True, s=s))
    q = q[:, :, 0]
    assert torch.equal(hb().cache_decode(q.expand(2, -1, -1), cache, table, kv, s=s), hb().cache_decode(q.repeat(2, 1, 1), cache, table, kv, s=s))


def test_two_captured_graphs_with_one_workspace():
    """Replayed one after the other on a stream, in any order; lengths change between replays."""
    Hq, Hkv, d, lens = 8, 2, 128, [900, 130]
    cache, table, k, v, s, inv_s = make_cache(lens, Hkv, d, "bf16")
    kv = ints(lens)
    q1 = torch.randn((2, Hq, d), device=DEV).bfloat16()
    q40 = torch.randn((2, Hq, 40, d), device=DEV).bfloat16()
    w = torch.zeros(table.shape, device=DEV)
    nbytes = max(hb().cache_decode_workspace_bytes(cache, 2, table.shape[1], Hq, with_page_weight=True),
                 hb().cache_attention_workspace_bytes(cache, 2, table.shape[1], Hq, 40))
    ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    outs = [torch.empty_like(q1), torch.empty_like(q40)]
    calls = [lambda: hb().cache_decode(q1, cache, table, kv, s=s, out=outs[0], page_weight_out=w, workspace=ws),
             lambda: hb().cache_attention(q40, cache, table, kv, True, s=s, out=outs[1], workspace=ws)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for call in calls:
            call()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                call()
            graphs.append(graph)
    torch.cuda.current_stream().wait_stream(side)
    for x in ([900, 130], [64, 100], [0, 129], [513, 1]):
        kv.copy_(ints(x))
        want = [hb().cache_decode(q1, cache, table, kv, s=s), hb().cache_attention(q40, cache, table, kv, True, s=s)]
        for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
            for o in outs:
                o.fill_(9)
            for i in order:
                graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_a_bad_page_does_not_hide_an_expired_wait():
    """Several calls may share a status word that is read at the end: what says that outputs are missing stays in it."""
    lens = [200, 130]
    cache, table, k, v, s, inv_s = make_cache(lens, 2, 128, "bf16")
    bad = table.clone()
    bad[0, 1] = -7
    q, kv, wrong = torch.randn((2, 4, 128), device=DEV).bfloat16(), ints(lens), ints([-1, 130])
    calls = [lambda st: hb().cache_decode(q, cache, bad, kv, d_status=st), lambda st: hb().cache_decode(q, cache, table, wrong, d_status=st),
             lambda st: hb().cache_attention(q[:, :, None].repeat(1, 1, 40, 1), cache, bad, kv, False, d_status=st),
             lambda st: hb().cache_read(cache, bad, kv, 200, d_status=st), lambda st: hb().cache_evict(table, wrong, torch.zeros(table.shape, device=DEV), 2, d_status=st),
             lambda st: hb().cache_append(cache, k[:, :, :1].to(DEV), v[:, :, :1].to(DEV), table, wrong, d_status=st)]
    for before, after in ((0, 1), (6, 6), (6 + 16 * 7, 6 + 16 * 7)):
        for call in calls:
            status = torch.full((1,), before, dtype=torch.int32, device=DEV)
            call(status)
            assert status.item() == after
