"""Paged HIF4 cache on the GPU: append byte for byte against the oracle's quantizer, attention against FP64 on the values that the
pages stand for, eviction against sorting, and a run of all of them together."""
import math
import random

import numpy as np
import pytest
import torch

from tests import cache_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def hb():
    from paper_2607_04302_b200 import binding
    return binding


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def make_cache(lens, Hkv, d, dtype, seed=0, spare=2, gain=None):
    """A cache with sequences of these lengths from random keys and values, its table, and k, v, inv_s."""
    gen = torch.Generator().manual_seed(seed)
    n = max(max(lens), 1)
    B = len(lens)
    k, v = torch.randn((B, Hkv, n, d), generator=gen), torch.randn((B, Hkv, n, d), generator=gen)
    s = torch.rand((Hkv, d), generator=gen) + 0.5
    s[:, 3] *= 4
    k[..., 3] *= 16
    k, v = k.to(DT[dtype]), v.to(DT[dtype])
    need = [(x + 63) // 64 for x in lens]
    cache = hb().alloc_cache(sum(need) + spare, Hkv, d, DT[dtype], DEV, B)
    cache.pages.random_(0, 256, generator=torch.Generator(DEV).manual_seed(seed))       # old contents
    cache.v_tail.normal_(generator=torch.Generator(DEV).manual_seed(seed + 1))
    perm = torch.randperm(sum(need) + spare, generator=gen).int()
    table = torch.full((B, max(need) + 1), -1, dtype=torch.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = perm[at:at + m]
        at += m
    table = table.to(DEV)
    inv_s = (1 / s).to(DEV)
    hb().cache_append(cache, k.to(DEV), v.to(DEV), table, ints(lens), n_new=ints(lens), inv_s=inv_s)
    return cache, table, k, v, s.to(DEV), inv_s


def smoothed(k, inv_s, h):
    return ref.round_in(k.double() * inv_s[h].double().cpu(), k.dtype)


def check_pages(cache, table, k, v, inv_s, lens):
    """Every page byte that belongs to a token, and V's whole groups."""
    pages = cache.pages.cpu().numpy()
    Hkv, d = k.shape[1], k.shape[3]
    for b, n in enumerate(lens):
        for j in range((n + 63) // 64):
            rows = min(64, n - 64 * j)
            for h in range(Hkv):
                kk = torch.zeros(64, d, dtype=torch.float64)
                vv = torch.zeros(64, d, dtype=torch.float64)
                kk[:rows] = smoothed(k[b, h, 64 * j:64 * j + rows], inv_s, h)
                vv[:rows] = v[b, h, 64 * j:64 * j + rows].double()
                want, got = ref.page_bytes(kk.numpy(), vv.numpy()), pages[int(table[b, j]), h]
                G = d // 64
                for lo, width in ((0, d // 2), (32 * d, 4 * G), (36 * d, G)):
                    assert np.array_equal(got[lo:lo + rows * width], want[lo:lo + rows * width]), (b, j, h, lo)
                assert np.array_equal(got[37 * d:], want[37 * d:]), (b, j, h)
        if n % 64:
            assert torch.equal(cache.v_tail[b, :, :n % 64].cpu(), v[b, :, n - n % 64:n])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,Hkv", [(64, 3), (128, 2), (256, 1)])
def test_append_matches_the_oracle(d, Hkv, dtype):
    lens = [1, 0, 63, 64, 65, 200]
    cache, table, k, v, s, inv_s = make_cache(lens, Hkv, d, dtype)
    check_pages(cache, table, k, v, inv_s, lens)


def test_append_in_pieces_equals_one_append():
    """Chunks that begin and end anywhere, single tokens among them, other tail slots; rows of other pages stay."""
    H, d, dtype, lens = 2, 128, "bf16", [261, 70, 5]
    whole, table, k, v, s, inv_s = make_cache(lens, H, d, dtype)
    cache = hb().alloc_cache(whole.pages.shape[0], H, d, DT[dtype], DEV, 7)
    cache.pages.fill_(0x5A)
    slots = ints([6, 0, 3])
    rng, have = random.Random(3), [0, 0, 0]
    kd, vd = k.to(DEV), v.to(DEV)
    while have != lens:
        new = [min(l - h, rng.choice([0, 1, 1, 7, 64, 90])) for l, h in zip(lens, have)]
        n = max(new + [1]) + 2
        kn, vn = torch.zeros(3, H, n, d, dtype=DT[dtype], device=DEV), torch.zeros(3, H, n, d, dtype=DT[dtype], device=DEV)
        for b in range(3):
            kn[b, :, :new[b]], vn[b, :, :new[b]] = kd[b, :, have[b]:have[b] + new[b]], vd[b, :, have[b]:have[b] + new[b]]
        have = [h + x for h, x in zip(have, new)]
        hb().cache_append(cache, kn, vn, table, ints(have), n_new=ints(new), inv_s=inv_s, tail_slots=slots)
    moved = torch.stack([cache.v_tail[6], cache.v_tail[0], cache.v_tail[3]])
    check_pages(hb().PagedCache(cache.pages, moved), table, k, v, inv_s, lens)
    used = set(table[table >= 0].tolist())
    free = [p for p in range(cache.pages.shape[0]) if p not in used]
    assert (cache.pages[free] == 0x5A).all()


def test_append_and_read_take_strides_and_leave_other_rows():
    """k and v as slices of a fused projection [B, n, (2 Hkv) d]; the values come back; rows behind the end are left alone."""
    B, H, n, d = 3, 4, 100, 64
    gen = torch.Generator().manual_seed(5)
    x = torch.randn((B, n, 2 * H, d), generator=gen).half().to(DEV)
    k, v = x[:, :, :H].transpose(1, 2), x[:, :, H:].transpose(1, 2)
    lens = [100, 64, 37]
    table = torch.arange(6, dtype=torch.int32, device=DEV).view(3, 2)
    cache = hb().alloc_cache(6, H, d, torch.float16, DEV, B)
    hb().cache_append(cache, k, v, table, ints(lens), n_new=ints(lens))
    check_pages(cache, table, k.cpu(), v.cpu(), torch.ones(H, d), lens)
    for dt in (hb().BF16, hb().F32):
        out = [torch.full((B, H, 50, d), 7.0, dtype={hb().BF16: torch.bfloat16, hb().F32: torch.float32}[dt], device=DEV) for _ in range(2)]
        start = [60, 10, 0]
        hb().cache_read(cache, table, ints(lens), 50, start=ints(start), out=out)
        pages = cache.pages.cpu()
        for b in range(B):
            for h in range(H):
                K, V = ref.sequence(pages, table[b].cpu(), lens[b], h)
                m = min(50, lens[b] - start[b])
                assert torch.equal(out[0][b, h, :m].double().cpu(), K[start[b]:start[b] + m])
                assert torch.equal(out[1][b, h, :m].double().cpu(), V[start[b]:start[b] + m])
        assert all((o[2, :, 37:] == 7).all() and (o[0, :, 40:] == 7).all() for o in out)


def test_append_extreme_values():
    """Groups at both ends of the scale's range, zeros, an infinity (saturates) and a NaN (stored as zero)."""
    d = 128
    e = torch.linspace(-60, 30, 64)[:, None]
    gen = torch.Generator().manual_seed(2)
    k = (torch.randn((64, d), generator=gen) * torch.exp2(e)).bfloat16()
    v = (torch.randn((d, 64), generator=gen) * torch.exp2(torch.linspace(-60, 30, d))[:, None]).T.contiguous().bfloat16()
    k[5] = 0
    v[:, 9] = 0
    cache = hb().alloc_cache(1, 1, d, torch.bfloat16, DEV, 1)
    table, lens = ints([[0]]), ints([64])
    hb().cache_append(cache, k[None, None].to(DEV), v[None, None].to(DEV), table, lens)
    assert np.array_equal(cache.pages[0, 0].cpu().numpy(), ref.page_bytes(k.double().numpy(), v.double().numpy()))
    k[7, 3], v[8, 11], k[9, 70], v[20, 30] = math.inf, -math.inf, math.nan, math.nan
    hb().cache_append(cache, k[None, None].to(DEV), v[None, None].to(DEV), table, lens)
    K, V = ref.values(cache.pages[0, 0].cpu().numpy())
    top = 7 * 1.75 * 2.0 ** 15
    assert K[7, 3] == top and V[8, 11] == -top and K[9, 70] == 0 and V[20, 30] == 0
    assert np.isfinite(K).all() and np.isfinite(V).all()


def check_attention(out, r, d, p_bits=11):
    err = (out.double().cpu() - r.out).abs()
    tol = ref.tolerance(r, d, out.dtype, p_bits)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("Hq,Hkv,d,dtype,lens", [
    (1, 1, 128, "bf16", [1]), (4, 1, 128, "fp16", [64]), (32, 8, 128, "bf16", [100]), (8, 8, 64, "bf16", [63, 65, 0, 1, 700]),
    (12, 4, 64, "fp16", [0, 0, 129]), (16, 8, 256, "bf16", [200, 1, 320]), (10, 2, 128, "fp16", [3000, 17]),
    (28, 4, 64, "bf16", [500, 40]), (9, 1, 256, "fp16", [130]), (24, 2, 128, "bf16", [333, 5000]), (40, 1, 128, "bf16", [77, 0]),
    (5, 5, 128, "bf16", [64, 128, 192, 256, 1, 2, 3, 4, 0, 1000, 70, 64, 64])])
def test_decode_matches_fp64(Hq, Hkv, d, dtype, lens):
    cache, table, k, v, s, inv_s = make_cache(lens, Hkv, d, dtype, seed=len(lens))
    B = len(lens)
    gen = torch.Generator().manual_seed(11)
    q = (torch.randn((B, Hq, d), generator=gen) * 2).to(DT[dtype])
    lse = torch.empty(B, Hq, device=DEV)
    w0 = torch.rand(table.shape, generator=gen).to(DEV)
    w1 = torch.full_like(w0, -3.0)
    out = hb().cache_decode(q.to(DEV), cache, table, ints(lens), s=s, lse=lse, page_weight=w0, page_weight_out=w1)
    r = ref.attend(q[:, :, None], cache.pages.cpu(), table.cpu(), lens, s.cpu())
    check_attention(out[:, :, None], r, d)
    lse_ref, weight = r.lse[..., 0], r.weight
    ds = ref.score_error(r.E[..., 0], d)
    empty = lse_ref == -math.inf
    assert torch.equal(lse.double().cpu() == -math.inf, empty)
    err = torch.where(empty, 0.0, (lse.double().cpu() - lse_ref).abs())
    assert (err <= ds + 2.0 ** -20 + 2.0 ** -21 * lse_ref.abs().nan_to_num(0, 0, 0)).all()
    # every p and every sum off by a factor 1 + eps, and the sum over the heads 2^-20
    eps = 2 * (torch.expm1(ds).amax(1, keepdim=True) + 2.0 ** -20) + 2.0 ** -20
    got = w1.double().cpu()
    for b, n in enumerate(lens):
        m = (n + 63) // 64
        tot = w0[b, :m].double().cpu() + weight[b, :m]
        assert ((got[b, :m] - tot).abs() <= eps[b] * weight[b, :m] + 2.0 ** -23 * tot).all()
        assert (got[b, m:] == -3).all()


def test_decode_options():
    """A head map, strides, a scale, FP32 output, a preallocated workspace; in-place page weights; equal calls, equal bits."""
    Hq, Hkv, d, lens = 7, 3, 128, [300, 64]
    cache, table, k, v, s, inv_s = make_cache(lens, Hkv, d, "bf16")
    q_to_kv = [2, 0, 1, 2, 2, 0, 2]
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((2, Hq, 3 * d), generator=gen).bfloat16().to(DEV)
    q = x[..., d:2 * d]
    out = torch.empty(2, Hq, d, device=DEV)
    ws = torch.empty(hb().cache_decode_workspace_bytes(cache, 2, table.shape[1], Hq, q_to_kv, True), dtype=torch.uint8, device=DEV)
    ws.fill_(255)
    w = torch.zeros(table.shape, device=DEV)
    hb().cache_decode(q, cache, table, ints(lens), out=out, softmax_scale=0.3, q_to_kv=q_to_kv, workspace=ws, page_weight=w, page_weight_out=w)
    r = ref.attend(q.cpu()[:, :, None], cache.pages.cpu(), table.cpu(), lens, None, q_to_kv=q_to_kv, scale=0.3)
    check_attention(out[:, :, None], r, d)
    assert torch.allclose(w.double().cpu(), r.weight, rtol=1e-4, atol=0)
    first = out.clone()
    hb().cache_decode(q, cache, table, ints(lens), out=out, softmax_scale=0.3, q_to_kv=q_to_kv, workspace=ws)
    assert torch.equal(out, first)


@pytest.mark.parametrize("lens,B", [([20000], 1), ([9000, 64, 12000, 1], 4)])
def test_decode_long(lens, B):
    """Segments that many CTAs share."""
    cache, table, k, v, s, inv_s = make_cache(lens, 2, 128, "bf16")
    q = (torch.randn((B, 8, 128), generator=torch.Generator().manual_seed(4)) * 3).bfloat16()
    out = hb().cache_decode(q.to(DEV), cache, table, ints(lens), s=s)
    r = ref.attend(q[:, :, None], cache.pages.cpu(), table.cpu(), lens, s.cpu())
    check_attention(out[:, :, None], r, 128)


@pytest.mark.parametrize("Hq,Hkv,d,dtype", [(8, 1, 256, "bf16"), (16, 2, 256, "fp16"), (14, 2, 64, "fp16"), (24, 2, 64, "bf16"), (30, 2, 128, "fp16")])
def test_decode_long_of_every_width(Hq, Hkv, d, dtype):
    """Segments within a consumer, across consumers and across CTAs, of each head dimension and block of rows, with page weights; then
    with a page that is not there."""
    lens = [9000, 130, 3000, 64]
    cache, table, k, v, s, inv_s = make_cache(lens, Hkv, d, dtype, seed=d)
    q = (torch.randn((4, Hq, d), generator=torch.Generator().manual_seed(d)) * 2).to(DT[dtype])
    w = torch.full(table.shape, 7.0, device=DEV)

    def check(out, table, lens, rows, cols):
        r = ref.attend(q[rows][:, :, None], cache.pages.cpu(), table.cpu(), lens, s.cpu())
        check_attention(out[rows][:, :, None], r, d)
        ds = ref.score_error(r.E[..., 0], d)
        eps = 2 * (torch.expm1(ds).amax(1, keepdim=True) + 2.0 ** -20) + 2.0 ** -20          # as in test_decode_matches_fp64
        got = w[rows][:, cols].double().cpu()
        for b, n in enumerate(lens):
            m = (n + 63) // 64
            assert ((got[b, :m] - r.weight[b, :m]).abs() <= eps[b] * r.weight[b, :m] + 2.0 ** -23).all()

    out = hb().cache_decode(q.to(DEV), cache, table, ints(lens), s=s, page_weight_out=w)
    check(out, table, lens, [0, 1, 2, 3], list(range(table.shape[1])))
    assert (w[1, 3:] == 7).all() and (w[3, 1:] == 7).all()
    again = hb().cache_decode(q.to(DEV), cache, table, ints(lens), s=s)
    assert torch.equal(out, again)
    bad, status = table.clone(), torch.zeros(1, dtype=torch.int32, device=DEV)
    bad[0, 70] = -1
    out = hb().cache_decode(q.to(DEV), cache, bad, ints(lens), s=s, page_weight_out=w, d_status=status)
    cols = [i for i in range(table.shape[1]) if i != 70]
    check(out, table[:1, cols], [9000 - 64], [0], cols)
    assert status.item() == 1 and w[0, 70] == 0 and torch.equal(out[1:], again[1:])


def test_bad_lengths_and_pages_are_left_out():
    """Found on the device: the sequence (page) is left out, the status word says so, the others are as usual."""
    lens = [200, 130, 64]
    cache, table, k, v, s, inv_s = make_cache(lens, 2, 128, "bf16")
    q = torch.randn((3, 4, 128), generator=torch.Generator().manual_seed(4)).bfloat16()
    good = hb().cache_decode(q.to(DEV), cache, table, ints(lens))
    for bad_len, bad_page in ((-1, None), (64 * table.shape[1] + 1, None), (None, 10 ** 6), (None, -5)):
        t, l = table.clone(), ints(lens)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        if bad_len is not None:
            l[1] = bad_len
        else:
            t[1, 1] = bad_page
        out = hb().cache_decode(q.to(DEV), cache, t, l, d_status=status)
        assert status.item() == 1
        assert torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])
        if bad_len is not None:
            assert (out[1] == 0).all()
        else:                                            # the page's 64 tokens are missing
            keep = t[1:2, [0, 2]].contiguous()
            again = hb().cache_decode(q[1:2].to(DEV), cache, keep, ints([66]))
            assert torch.allclose(out[1].float(), again[0].float(), rtol=0, atol=0.02)
        before = cache.pages.clone()
        status.zero_()
        hb().cache_append(cache, k[:, :, :64].to(DEV), v[:, :, :64].to(DEV), t, l, n_new=ints([0, 64, 0]), d_status=status)
        assert status.item() == 1
        ids = [int(x) for x in table[1] if x >= 0]
        others = [p for p in range(cache.pages.shape[0]) if p not in ids]
        assert torch.equal(cache.pages[others], before[others])
        cache.pages.copy_(before)
        status.zero_()
        r = hb().cache_evict(t, l, torch.rand(t.shape, device=DEV), 2, d_status=status)
        assert status.item() == (1 if bad_len is not None else 0)
        if bad_len is not None:
            assert r.n_freed[1].item() == 0 and torch.equal(r.block_table[1], t[1]) and r.kv_lens[1].item() == bad_len


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB: its last pages."""
    H, d = 8, 256
    n_pages = (1 << 32) // (H * 74 * d) + 40
    pages = torch.empty((n_pages, H, 74 * d), dtype=torch.uint8, device=DEV)
    cache = hb().PagedCache(pages, torch.zeros((1, H, 64, d), dtype=torch.bfloat16, device=DEV))
    table = torch.arange(n_pages - 5, n_pages, dtype=torch.int32, device=DEV)[None].contiguous()
    gen = torch.Generator().manual_seed(0)
    k, v = (torch.randn((1, H, 300, d), generator=gen).bfloat16() for _ in range(2))
    hb().cache_append(cache, k.to(DEV), v.to(DEV), table, ints([300]))
    small = hb().PagedCache(pages[-5:].clone(), None)
    q = torch.randn((1, 16, d), generator=gen).bfloat16()
    out = hb().cache_decode(q.to(DEV), cache, table, ints([300]))
    r = ref.attend(q[:, :, None], small.pages.cpu(), torch.arange(5)[None], [300])
    check_attention(out[:, :, None], r, d)


@pytest.mark.parametrize("Hq,Hkv,d,N,dtype,causal,lens", [
    (4, 2, 128, 2, "bf16", True, [1, 2, 130, 0]), (6, 2, 64, 5, "fp16", False, [3, 64, 0, 200]), (8, 2, 128, 70, "bf16", True, [20, 70, 300]),
    (2, 2, 256, 33, "fp16", True, [100, 32]), (3, 1, 64, 130, "bf16", False, [65, 400]), (12, 4, 128, 129, "fp16", True, [129, 257]),
    (4, 4, 256, 200, "bf16", False, [500]), (1, 1, 128, 1, "bf16", True, [77]), (16, 2, 128, 40, "bf16", True, [64, 1000, 41])])
def test_attention_matches_fp64(Hq, Hkv, d, N, dtype, causal, lens):
    cache, table, k, v, s, inv_s = make_cache(lens, Hkv, d, dtype, seed=N)
    q = (torch.randn((len(lens), Hq, N, d), generator=torch.Generator().manual_seed(N)) * 2).to(DT[dtype])
    out = hb().cache_attention(q.to(DEV), cache, table, ints(lens), causal, s=s)
    r = ref.attend(q, cache.pages.cpu(), table.cpu(), lens, s.cpu(), causal=causal)
    check_attention(out, r, d, P_BITS[dtype])
    assert (out.cpu()[r.lse == -math.inf] == 0).all()


# bits of P in the product with V: BF16 keeps 8 (half a step: 2^-8), its two-term form and FP16 11 or more
P_BITS = {"bf16": 8, "fp16": 11}


@pytest.mark.parametrize("B,P,keep,first,last", [(1, 1, 1, 0, 1), (5, 40, 11, 1, 2), (3, 64, 64, 3, 3), (2, 33, 2, 1, 1), (4, 3000, 700, 2, 16),
                                                 (2, 1025, 1024, 0, 1)])
def test_evict_matches_sorting(B, P, keep, first, last):
    rng = np.random.default_rng(P)
    table = np.stack([rng.permutation(10 * P)[:P] for _ in range(B)]).astype(np.int32)
    lens = np.array([64 * P - 5] + [int(rng.integers(0, 64 * P + 1)) for _ in range(B - 1)], np.int32)
    weight = rng.choice(np.array([0.0, -0.0, 1.0, 0.25, 7.5, -2.0, np.inf, -np.inf, np.nan], np.float32), (B, P))
    mixed = rng.random((B, P)).astype(np.float32)
    weight = np.where(rng.random((B, P)) < 0.5, weight, mixed).astype(np.float32)
    want = ref.evict(table, lens, weight, keep, first, last)
    t, l, w = torch.from_numpy(table).to(DEV), torch.from_numpy(lens).to(DEV), torch.from_numpy(weight).to(DEV)
    for in_place in (False, True):
        out = hb().alloc_evicted(t)
        if in_place:
            out.block_table, out.kv_lens, out.page_weight = t, l, w
        r = hb().cache_evict(t, l, w, keep, first, last, out=out)
        assert np.array_equal(r.block_table.cpu().numpy(), want["table"])
        assert r.kv_lens.tolist() == want["lens"] and r.n_freed.tolist() == want["n"]
        assert np.array_equal(r.page_weight.cpu().numpy(), want["weight"], equal_nan=True)
        assert np.array_equal(r.freed.cpu().numpy(), want["freed"])


def test_evict_whole_classes_of_weights():
    """The border between what stays and what goes falls between classes of equal weights, inside one, and among NaN; weights that
    differ in their first, in their last and in no digit."""
    P = 200
    low = np.arange(P, dtype=np.uint32) + 0x3F800000                       # differ in their last bits
    sets = [np.repeat(np.float32([1, 2, 3, 4]), 50), low.view(np.float32), (low * 256).view(np.float32), np.zeros(P, np.float32),
            np.where(np.arange(P) % 2, np.nan, 1.0).astype(np.float32), np.full(P, np.nan, np.float32), np.repeat(np.float32([-1, -0.0, 0.0, 1]), 50)]
    weight = np.stack(sets).astype(np.float32)
    B = len(sets)
    table, lens = np.tile(np.arange(P, dtype=np.int32), (B, 1)), np.full(B, 64 * P, np.int32)
    t, l, w = torch.from_numpy(table).to(DEV), torch.from_numpy(lens).to(DEV), torch.from_numpy(weight).to(DEV)
    for keep in (2, 3, 51, 52, 53, 101, 102, 103, 150, 151, 152, 199, 200):
        r, want = hb().cache_evict(t, l, w, keep, 1, 1), ref.evict(table, lens, weight, keep, 1, 1)
        assert np.array_equal(r.block_table.cpu().numpy(), want["table"]) and r.kv_lens.tolist() == want["lens"]
        assert np.array_equal(r.freed.cpu().numpy(), want["freed"]) and r.n_freed.tolist() == want["n"], keep


def test_serving_run():
    """Prompt, twenty steps with page weights, an eviction, more steps over the shorter tables, a second chunk: each against FP64."""
    Hq, Hkv, d = 8, 2, 128
    lens = [150, 700]
    cache, table, k, v, s, inv_s = make_cache(lens, Hkv, d, "bf16", spare=14)
    spare = [p for p in range(cache.pages.shape[0]) if p not in set(table[table >= 0].tolist())]
    table = torch.cat([table, torch.full((2, 6), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
    gen = torch.Generator().manual_seed(9)
    weight = torch.zeros(table.shape, device=DEV)
    total = torch.zeros(table.shape, dtype=torch.float64)

    def step(n, causal_attention=False):
        nonlocal lens
        lens = [x + n for x in lens]
        for b, x in enumerate(lens):
            for j in range((x + 63) // 64):
                if table[b, j] < 0:
                    table[b, j] = spare.pop()
        kn, vn = (torch.randn((2, Hkv, n, d), generator=gen).bfloat16() for _ in range(2))
        q = (2 * torch.randn((2, Hq, n, d), generator=gen)).bfloat16()
        hb().cache_append(cache, kn.to(DEV), vn.to(DEV), table, ints(lens), inv_s=inv_s)
        r = ref.attend(q, cache.pages.cpu(), table.cpu(), lens, s.cpu(), causal=True)
        if n == 1:
            out = hb().cache_decode(q[:, :, 0].contiguous().to(DEV), cache, table, ints(lens), s=s, page_weight=weight, page_weight_out=weight)
            total.add_(r.weight)
            check_attention(out[:, :, None], r, d)
        else:
            out = hb().cache_attention(q.to(DEV), cache, table, ints(lens), True, s=s)
            check_attention(out, r, d, 8)

    for _ in range(20):
        step(1)
    assert torch.allclose(weight.double().cpu(), total, rtol=1e-4, atol=1e-6)
    r = hb().cache_evict(table, ints(lens), weight, 6, 1, 2)
    want = ref.evict(table.cpu().numpy(), lens, weight.cpu().numpy(), 6, 1, 2)
    assert r.n_freed.tolist() == [0, 6] and np.array_equal(r.block_table.cpu().numpy(), want["table"])
    table, weight, lens = r.block_table, r.page_weight, r.kv_lens.tolist()
    spare += r.freed[1, :6].tolist()
    total = weight.double().cpu()
    for _ in range(3):
        step(1)
    step(90)


def test_captured_step_is_replayed_with_other_lengths():
    """Append and decode captured once; tables and lengths change between replays, on a stream of its own."""
    Hq, Hkv, d, lens = 4, 2, 128, [60, 130]
    cache, table, k, v, s, inv_s = make_cache(lens, Hkv, d, "bf16")
    table = torch.cat([table, table[:, :1] * 0 - 1], 1).contiguous()
    table[0, 1] = cache.pages.shape[0] - 1 if (cache.pages.shape[0] - 1) not in table.tolist()[1] else 0
    used = set(x for x in table.flatten().tolist() if x >= 0)
    assert len(used) == int((table >= 0).sum())
    kv = ints(lens)
    kn = torch.randn(2, Hkv, 1, d, device=DEV).bfloat16()
    vn, q = torch.randn_like(kn), torch.randn(2, Hq, d, device=DEV).bfloat16()
    out = torch.empty_like(q)
    w = torch.zeros(table.shape, device=DEV)

    def call():
        hb().cache_append(cache, kn, vn, table, kv, inv_s=inv_s)
        hb().cache_decode(q, cache, table, kv, s=s, out=out, page_weight=w, page_weight_out=w)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kv += 1
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(6):
        kv += 1
        for x in (kn, vn, q):
            x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        r = ref.attend(q.cpu()[:, :, None], cache.pages.cpu(), table.cpu(), kv.tolist(), s.cpu())
        check_attention(out[:, :, None], r, d)


def test_many_short_sequences():
    """More sequences than a warp or a block looks over at once; empty ones among them; page weights."""
    rng = random.Random(5)
    lens = [rng.choice([0, 1, 63, 64, 65, rng.randint(1, 200)]) for _ in range(301)]
    cache, table, k, v, s, inv_s = make_cache(lens, 2, 64, "fp16")
    q = torch.randn((len(lens), 6, 64), generator=torch.Generator().manual_seed(8)).half()
    w = torch.zeros(table.shape, device=DEV)
    out = hb().cache_decode(q.to(DEV), cache, table, ints(lens), s=s, page_weight_out=w)
    r = ref.attend(q[:, :, None], cache.pages.cpu(), table.cpu(), lens, s.cpu())
    check_attention(out[:, :, None], r, 64)
    assert torch.allclose(w.double().cpu(), r.weight, rtol=1e-4, atol=1e-6)
    out = hb().cache_attention(q[:40, :, None].repeat(1, 1, 70, 1).to(DEV), cache, table[:40].contiguous(), ints(lens[:40]), False, s=s)
    r = ref.attend(q[:40, :, None], cache.pages.cpu(), table[:40].cpu(), lens[:40], s.cpu())
    check_attention(out[:, :, 69:], r, 64)
    assert torch.equal(out[:, :, 0], out[:, :, 69])


@pytest.mark.parametrize("Hq,Hkv,d,N,dtype,causal,lens", [
    (8, 2, 64, 64, "fp16", True, [1500, 900]), (8, 2, 128, 64, "fp16", False, [2000, 10]), (2, 1, 256, 100, "bf16", True, [1700]),
    (2, 1, 256, 80, "fp16", False, [1300]), (4, 1, 128, 64, "bf16", True, [2500]), (2, 2, 128, 128, "bf16", False, [64, 65]),
    (1, 1, 64, 257, "bf16", True, [300]), (32, 2, 128, 16, "bf16", False, [1, 0, 640]), (3, 1, 128, 43, "bf16", True, [43])])
def test_attention_split_and_paired_tiles(Hq, Hkv, d, N, dtype, causal, lens):
    """Blocks shared out over their pages, both tiles on the same rows (an odd and an even number of pages, one page), partly empty tiles."""
    cache, table, k, v, s, inv_s = make_cache(lens, Hkv, d, dtype, seed=N)
    q = (torch.randn((len(lens), Hq, N, d), generator=torch.Generator().manual_seed(N)) * 2).to(DT[dtype])
    out = hb().cache_attention(q.to(DEV), cache, table, ints(lens), causal, s=s)
    r = ref.attend(q, cache.pages.cpu(), table.cpu(), lens, s.cpu(), causal=causal)
    check_attention(out, r, d, P_BITS[dtype])
    again = hb().cache_attention(q.to(DEV), cache, table, ints(lens), causal, s=s)
    assert torch.equal(out, again)


def test_attention_options():
    """A head map, strides, a scale, FP32 output, a dirty workspace; a missing page and a bad length."""
    Hq, Hkv, d, N, lens = 7, 3, 128, 40, [300, 64, 130]
    cache, table, k, v, s, inv_s = make_cache(lens, Hkv, d, "bf16")
    q_to_kv = [2, 0, 1, 2, 2, 0, 2]
    x = torch.randn((3, N, Hq, 2 * d), generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    q = x[..., d:].transpose(1, 2)
    out = torch.empty(3, Hq, N, d, device=DEV)
    ws = torch.full((hb().cache_attention_workspace_bytes(cache, 3, table.shape[1], Hq, N, q_to_kv=q_to_kv),), 255, dtype=torch.uint8, device=DEV)
    hb().cache_attention(q, cache, table, ints(lens), True, out=out, softmax_scale=0.3, q_to_kv=q_to_kv, workspace=ws)
    r = ref.attend(q.cpu(), cache.pages.cpu(), table.cpu(), lens, None, causal=True, q_to_kv=q_to_kv, scale=0.3)
    check_attention(out, r, d, 8)
    t, l, status = table.clone(), ints([300, 64, 10 ** 6]), torch.zeros(1, dtype=torch.int32, device=DEV)
    t[0, 1] = 10 ** 6
    bad = hb().cache_attention(q, cache, t, l, False, softmax_scale=0.3, q_to_kv=q_to_kv, d_status=status)
    good = hb().cache_attention(q, cache, table, ints(lens), False, softmax_scale=0.3, q_to_kv=q_to_kv)
    assert status.item() == 1 and torch.equal(bad[1], good[1]) and (bad[2] == 0).all()
    r = ref.attend(q[:1].cpu(), cache.pages.cpu(), table[:1, [0, 2, 3, 4]].cpu(), [300 - 64], None, q_to_kv=q_to_kv, scale=0.3)
    check_attention(bad[:1], r, d, 8)


@pytest.mark.parametrize("N", [1, 3, 40])
def test_not_a_number_stays_in_its_row(N):
    """A query row with a NaN, or with an infinity, spoils itself only."""
    lens = [200, 70]
    cache, table, k, v, s, inv_s = make_cache(lens, 2, 128, "bf16")
    q = torch.randn((2, 8, N, 128), generator=torch.Generator().manual_seed(4)).bfloat16()
    call = lambda q: hb().cache_attention(q.to(DEV), cache, table, ints(lens), False).cpu()
    clean = call(q)
    q[0, 3, N - 1, 7], q[1, 5, 0, 9] = math.nan, math.inf
    out = call(q)
    assert out[0, 3, N - 1].isnan().all() and out[1, 5, 0].isnan().all()
    spoilt = torch.zeros(2, 8, N, dtype=torch.bool)
    spoilt[0, 3, N - 1] = spoilt[1, 5, 0] = True
    assert torch.equal(out[~spoilt], clean[~spoilt])


def test_calls_on_two_streams_at_once():
    """Two streams, a workspace each (torch gives every call its own), the same cache."""
    lens = [3000, 500]
    cache, table, k, v, s, inv_s = make_cache(lens, 2, 128, "bf16")
    q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(4)).bfloat16().to(DEV)
    qn = torch.randn((2, 8, 50, 128), generator=torch.Generator().manual_seed(5)).bfloat16().to(DEV)
    one, many = hb().cache_decode(q, cache, table, ints(lens)), hb().cache_attention(qn, cache, table, ints(lens), False)
    kv = ints(lens)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(20):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(hb().cache_decode(q, cache, table, kv) if i == 0 else hb().cache_attention(qn, cache, table, kv, False))
    torch.cuda.synchronize()
    assert all(torch.equal(x, one) for x in got[0]) and all(torch.equal(x, many) for x in got[1])


def test_rows_of_other_sequences_stay():
    """A batch whose last rows are padding: tables of -1, length 0, no new tokens: pages, tails and page weights stay as they were."""
    lens = [100, 0, 0]
    cache, table, k, v, s, inv_s = make_cache(lens, 2, 64, "fp16")
    pages, tail = cache.pages.clone(), cache.v_tail.clone()
    w = torch.full(table.shape, 0.5, device=DEV)
    q = torch.randn((3, 4, 64), generator=torch.Generator().manual_seed(4)).half().to(DEV)
    kn = torch.randn((3, 2, 1, 64), generator=torch.Generator().manual_seed(6)).half().to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    hb().cache_append(cache, kn, kn, table, ints([101, 0, 0]), n_new=ints([1, 0, 0]), d_status=status)
    hb().cache_decode(q, cache, table, ints([101, 0, 0]), page_weight=w, page_weight_out=w, d_status=status)
    used = set(table[0, :2].tolist())
    rest = [p for p in range(pages.shape[0]) if p not in used]
    assert status.item() == 0 and torch.equal(cache.pages[rest], pages[rest]) and torch.equal(cache.v_tail[1:], tail[1:])
    assert torch.equal(cache.v_tail[0, :, :36], tail[0, :, :36]) and torch.equal(cache.v_tail[0, :, 37:], tail[0, :, 37:])
    assert (w[1:] == 0.5).all() and (w[0, 2:] == 0.5).all() and abs(float(w[0, :2].sum()) - 1.0 - 4) < 1e-4


def test_binding_refuses_tensors():
    cache, table, k, v, s, inv_s = make_cache([100], 2, 64, "fp16")
    q = torch.randn((1, 4, 64), device=DEV).half()
    bad = [dict(kv_lens=ints([100]).cpu()), dict(kv_lens=ints([100]).long()), dict(block_table=table.cpu()), dict(s=s.double()), dict(q=q.cpu()),
           dict(q=q[..., ::2]), dict(q=q.float()), dict(lse=torch.empty(4, device=DEV)), dict(out=torch.empty(1, 4, 32, device=DEV)),
           dict(page_weight_out=torch.zeros(1, 1, device=DEV))]
    for b in bad:
        args = dict(q=q, cache=cache, block_table=table, kv_lens=ints([100]), s=s)
        args.update(b)
        with pytest.raises((AssertionError, KeyError)):
            hb().cache_decode(**args)
    with pytest.raises(AssertionError):
        hb().cache_append(hb().PagedCache(cache.pages, None), k.to(DEV), v.to(DEV), table, ints([100]))
    with pytest.raises(hb().Hifa4Error):
        hb().cache_decode(q, cache, table, ints([100]), workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(hb().Hifa4Error):
        hb().cache_evict(table, ints([100]), torch.zeros(table.shape, device=DEV), 1, 1, 1)


def test_binding_refuses_host_status_words_and_unaligned_factors():
    cache, table, k, v, s, inv_s = make_cache([100], 2, 64, "fp16")
    q, kv, status = torch.randn((1, 4, 64), device=DEV).half(), ints([100]), torch.zeros(1, dtype=torch.int32)
    w = torch.zeros(table.shape, device=DEV)
    for call in (lambda: hb().cache_decode(q, cache, table, kv, d_status=status), lambda: hb().cache_read(cache, table, kv, 4, d_status=status),
                 lambda: hb().cache_attention(q[:, :, None], cache, table, kv, False, d_status=status),
                 lambda: hb().cache_append(cache, k.to(DEV), v.to(DEV), table, kv, d_status=status),
                 lambda: hb().cache_evict(table, kv, w, 1, 0, 1, d_status=status)):
        with pytest.raises(AssertionError):
            call()
    off = torch.ones(2 * 64 + 1, device=DEV)[1:].view(2, 64)
    out = [torch.empty(2 * 4 * 64 + 1, device=DEV)[1:].view(1, 2, 4, 64) for _ in range(2)]
    for call in (lambda: hb().cache_decode(q, cache, table, kv, s=off), lambda: hb().cache_append(cache, k.to(DEV), v.to(DEV), table, kv, inv_s=off),
                 lambda: hb().cache_attention(q[:, :, None], cache, table, kv, False, s=off), lambda: hb().cache_read(cache, table, kv, 4, out=out)):
        with pytest.raises(hb().Hifa4Error):
            call()


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "fp16"), (128, "bf16"), (256, "bf16")])
def test_between_other_kernels(d, dtype):
    """Calls that follow one another on a stream, each of which may start before the one before has ended: prefill attention, decode,
    attention of many tokens, appends, over and over, give what each gives alone."""
    lens = [1000, 130]
    cache, table, k, v, s, inv_s = make_cache(lens, 2, d, dtype)
    kv, kd, vd = ints(lens), k.to(DEV), v.to(DEV)
    gen = torch.Generator().manual_seed(8)
    qn = torch.randn((2, 4, 192, d), generator=gen).to(DT[dtype]).to(DEV)
    kp, vp = (torch.randn((2, 2, 192, d), generator=gen).to(DT[dtype]).to(DEV) for _ in range(2))
    q1 = qn[:, :, 0].contiguous()
    calls = [lambda: hb().cache_attention(qn, cache, table, kv, True, s=s), lambda: hb().attention_fwd_raw(qn, kp, vp, s, inv_s, True),
             lambda: hb().cache_attention(qn, cache, table, kv, False, s=s), lambda: hb().cache_decode(q1, cache, table, kv, s=s)]
    alone = []
    for call in calls:
        alone.append(call())
        torch.cuda.synchronize()
    for _ in range(10):
        for i in (0, 0, 1, 0, 2, 3, 1, 1, 3, 2):
            got = calls[i]()
            hb().cache_append(cache, kd, vd, table, kv, n_new=kv, inv_s=inv_s)           # (the same values again)
            again = calls[i]()
            assert torch.equal(got, alone[i]) and torch.equal(again, alone[i])


@pytest.mark.parametrize("counts", [(17, 0, 3), (1, 9, 0), (0, 0, 5)])
@pytest.mark.parametrize("N", [1, 2, 24])
def test_uneven_head_maps(counts, N):
    """KV heads with very different numbers of query heads, none among them: blocks of rows that do not exist."""
    q_to_kv = [g for g, n in enumerate(counts) for _ in range(n)]
    random.Random(1).shuffle(q_to_kv)
    lens = [900, 64, 0, 321] + [300] * 60
    cache, table, k, v, s, inv_s = make_cache(lens, 3, 64, "fp16")
    q = torch.randn((64, len(q_to_kv), N, 64), generator=torch.Generator().manual_seed(2)).half()
    out = torch.full(q.shape, 9.0, dtype=torch.float16, device=DEV)
    hb().cache_attention(q.to(DEV), cache, table, ints(lens), False, s=s, q_to_kv=q_to_kv, out=out)
    r = ref.attend(q, cache.pages.cpu(), table.cpu(), lens, s.cpu(), q_to_kv=q_to_kv)
    check_attention(out, r, 64)
    if N == 1:
        w = torch.zeros(table.shape, device=DEV)
        one = hb().cache_decode(q[:, :, 0].to(DEV), cache, table, ints(lens), s=s, q_to_kv=q_to_kv, page_weight_out=w)
        check_attention(one[:, :, None], r, 64)
        assert torch.allclose(w.double().cpu(), r.weight, rtol=1e-4, atol=1e-6)
