"""Failure path of the device waits of the paged cache's kernels: self-test instantiations (hifa4_selftest_cache_wait_timeout) in which
the first CTA's loader leaves a page out, so that a wait runs out and the CTA leaves.  Nothing hangs or faults; what does not depend
on that CTA is as in the ordinary call, and the next call is right."""
import pytest
import torch

from tests import cache_reference as ref
from tests.test_gpu_cache import DEV, check_attention, hb, ints, make_cache

pytestmark = pytest.mark.gpu


def shared_pages(B, n, Hkv, d):
    """B sequences of n tokens whose tables share the pages of a short one."""
    cache, table, k, v, s, inv_s = make_cache([64 * 40], Hkv, d, "bf16")
    pick = torch.randint(0, 40, (B, (n + 63) // 64 + 1), generator=torch.Generator().manual_seed(B))
    return cache, table[0].cpu()[pick].int().to(DEV).contiguous(), ints([n] * B)


def garbage(nbytes, kind):
    ws = torch.zeros((nbytes + 7) // 8 * 8, dtype=torch.uint8, device=DEV)
    if kind == "negative pairs":
        ws.view(torch.int32)[0::2], ws.view(torch.int32)[1::2] = -5, -3
    elif kind == "large pairs":
        ws.view(torch.int32)[0::2], ws.view(torch.int32)[1::2] = 3, 2 ** 30
    else:
        ws.fill_(255)
    return ws


@pytest.mark.parametrize("kind", ["ones", "negative pairs", "large pairs"])
@pytest.mark.parametrize("weight", [False, True])
def test_decode_gives_up_on_a_page(weight, kind):
    """The first consumer holds the beginning of the first sequence and head: its piece is missing in the CTA's join and in the join of
    the CTAs, and nobody records where the segment lies, so that the workspace's old contents are met there."""
    Hq, Hkv, d, B, n = 8, 4, 128, 4, 20000                   # 2 to 3 pages per consumer
    cache, table, kv = shared_pages(B, n, Hkv, d)
    q = torch.randn((B, Hq, d), generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    w_good, w = (torch.full(table.shape, 0.25, device=DEV) if weight else None for _ in range(2))
    good = hb().cache_decode(q, cache, table, kv, page_weight_out=w_good)
    ws = garbage(hb().cache_decode_workspace_bytes(cache, B, table.shape[1], Hq, with_page_weight=weight), kind)
    out, status = torch.full_like(q, 9.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    hb().selftest_cache_wait_timeout(q, cache, table, kv, status, out, ws, page_weight_out=w)
    torch.cuda.synchronize()
    assert status.item() == 6
    assert torch.equal(out[1:], good[1:]) and torch.equal(out[0, 2:], good[0, 2:])      # (heads 0 and 1 are those of the first KV head)
    assert not weight or torch.equal(w[1:], w_good[1:])
    status.zero_()
    again = hb().cache_decode(q, cache, table, kv, page_weight_out=w, workspace=ws, d_status=status)
    assert status.item() == 0 and torch.equal(again, good) and (not weight or torch.equal(w, w_good))
    r = ref.attend(q[:1, :, None].cpu(), cache.pages.cpu(), table[:1].cpu(), [n])
    check_attention(again[:1, :, None], r, d)


@pytest.mark.parametrize("Hq,Hkv,N,B,n,first", [(4, 2, 256, 40, 700, (0, 1)), (2, 2, 64, 2, 8000, (0, 0)), (2, 2, 300, 1, 8000, (0, 0))])
def test_attention_gives_up_on_a_page(Hq, Hkv, N, B, n, first):
    """A block of two tiles with a CTA of its own, and blocks that are shared out over their pages, with both tiles on the same rows,
    whose join reads what was never written."""
    d = 128
    cache, table, kv = shared_pages(B, n, Hkv, d)
    q = torch.randn((B, Hq, N, d), generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    good = hb().cache_attention(q, cache, table, kv, False)
    ws = garbage(hb().cache_attention_workspace_bytes(cache, B, table.shape[1], Hq, N), "ones")
    out, status = torch.full_like(q, 9.0), torch.zeros(1, dtype=torch.int32, device=DEV)
    hb().selftest_cache_wait_timeout(q, cache, table, kv, status, out, ws)
    torch.cuda.synchronize()
    assert status.item() == 6
    rest = torch.ones(B, Hq, dtype=torch.bool, device=DEV)
    rest[first] = False                                      # the head whose rows the first CTA has
    assert torch.equal(out[rest], good[rest])
    status.zero_()
    again = hb().cache_attention(q, cache, table, kv, False, workspace=ws, d_status=status)
    assert status.item() == 0 and torch.equal(again, good)


def test_refusals():
    cache, table, kv = shared_pages(1, 300, 2, 64)
    q = torch.zeros((1, 2, 64), device=DEV).bfloat16()
    ws, status = torch.empty(1 << 24, dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    with pytest.raises(hb().Hifa4Error):                     # d
        hb().selftest_cache_wait_timeout(q, cache, table, kv, status, torch.empty_like(q), ws)
    cache, table, kv = shared_pages(1, 300, 2, 128)
    for shape, st in (((1, 2, 128), None), ((1, 32, 128), status)):                       # no status word; 16 rows per KV head
        q = torch.zeros(shape, device=DEV).bfloat16()
        with pytest.raises(hb().Hifa4Error):
            hb().selftest_cache_wait_timeout(q, cache, table, kv, st, torch.empty_like(q), ws)
