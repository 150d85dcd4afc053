"""Serving from a 4-bit cache: what a program asks of the paged HIF4 key-value cache and of the attention that reads it.

Four operators, all reached through `paper_2607_04302_b200.binding`:
  append     cache_append: Smooth-QK and HIF4 quantization of new keys and values into the pages of a cache
             (then cache_read, which gives back the values that the cache now holds for them)
  step       cache_append of one token to every sequence, then cache_decode over the sequence with it
  decode     cache_decode: attention of one new token over the cache; optionally adds each page's share of the attention
             weight to a running total, and gives the logarithm of the softmax sum
  evict      cache_evict: the pages with the least accumulated weight leave the block table
  attention  cache_attention: many query tokens over the cache, all keys (cross attention to an encoder's states) or those
             up to their own position (the next chunk of a prompt)

A page holds 64 tokens of every KV head; a head's part has 74 d bytes, groups of 64 values as in include/hifa4.h (along
d for K, along the page's tokens for V), nibble = 8 + signed code:
  K codes   [64][4][d/64][2] words: units 2p, 2p+1 (8 elements each) of group G at [token][p][G]; element e in nibble e
  K shifts  [64][d/64] words: micro-exponent (0..2) of 4-element subgroup 2u+r in bits 16r+2u, +1
  K scales  [64][d/64] bytes: E6M2 codes
  V codes   [d][8] words: word 2i+h holds tokens 16i+4h+(0..3) in nibbles 0..3 and 16i+8+4h+(0..3) in nibbles 4..7
  V shifts  [d] words: that of the 4 tokens in nibbles 4r.. of word w in bits 16r+2w, +1
  V scales  [d] bytes"""
import math
import random

import numpy as np
import torch

own = False

_DT = {"fp16": torch.float16, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ cases
def _step(B, Hq, Hkv, d, lo, hi, dtype, mix=0):
    return dict(kind="step", B=B, Hq=Hq, Hkv=Hkv, d=d, lo=lo, hi=hi, dtype=dtype, mix=mix)


def _decode(B, Hq, Hkv, d, lo, hi, dtype, weight=False, lse=False, mix=0):
    return dict(kind="decode", B=B, Hq=Hq, Hkv=Hkv, d=d, lo=lo, hi=hi, dtype=dtype, weight=weight, lse=lse, mix=mix)


def _append(B, Hkv, d, lo, hi, start, dtype, smooth, mix=0):
    return dict(kind="append", B=B, Hkv=Hkv, d=d, lo=lo, hi=hi, start=start, dtype=dtype, smooth=smooth, mix=mix)


def _evict(B, pages, keep, first, last, mix=0):
    return dict(kind="evict", B=B, pages=pages, keep=keep, first=first, last=last, mix=mix)


def _attention(B, Hq, Hkv, d, N, lo, hi, causal, dtype, mix=0):
    return dict(kind="attention", B=B, Hq=Hq, Hkv=Hkv, d=d, N=N, lo=lo, hi=hi, causal=causal, dtype=dtype, mix=mix)


def listed():
    cases = {
        # the smallest step of one short dialogue: latency and launches count
        "step-1-short": _step(1, 32, 8, 128, 100, 100, "bf16"),
        # a serving batch takes one token further, sequences of all lengths
        "step-32-ragged": _step(32, 32, 8, 128, 17, 4097, "bf16"),
        # one long document, one token: the cache's length is all there is to split
        "decode-1-32k": _decode(1, 32, 8, 128, 32768, 32768, "bf16"),
        # a batch in the middle of its answers, with the weights that an eviction policy gathers
        "decode-64-ragged": _decode(64, 32, 8, 128, 1, 8192, "bf16", weight=True),
        # the largest: a full card of long sequences
        "decode-64-16k": _decode(64, 32, 8, 128, 12000, 16384, "bf16"),
        # Gemma2-9B-shaped heads, FP16, parts that are joined with another device's
        "decode-8-d256": _decode(8, 16, 8, 256, 5000, 8192, "fp16", lse=True),
        # a 32K prompt goes into the cache
        "append-32k-prompt": _append(1, 8, 128, 32768, 32768, 0, "bf16", True),
        # chunks of different lengths behind what a batch holds already, d = 64, FP16
        "append-16-chunks": _append(16, 4, 64, 1, 512, 1024, "fp16", False),
        # a small batch's tables shrink to a window of the heaviest pages
        "evict-4": _evict(4, 70, 32, 1, 2),
        # a large batch with long tables
        "evict-256-long": _evict(256, 2048, 512, 2, 16),
        # cross attention of a short target to an encoder's states of other lengths, d = 64
        "cross-8-short": _attention(8, 12, 12, 64, 77, 200, 1500, False, "fp16"),
        # the next 1024 tokens of four long prompts
        "chunk-4-1k": _attention(4, 32, 8, 128, 1024, 5001, 8192, True, "bf16"),
    }
    return [dict(c, name=n) for n, c in cases.items()]


_HEADS = [(1, 1), (4, 1), (8, 8), (12, 4), (12, 12), (14, 2), (16, 8), (28, 4), (32, 8), (40, 8)]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["step", "decode", "decode", "append", "evict", "attention", "attention"])
    mix = rng.randrange(1 << 30)
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    d = rng.choice([64, 128, 128, 128, 256])
    Hq, Hkv = rng.choice(_HEADS)
    if kind == "evict":
        B, pages = _log_int(rng, 1, 256), _log_int(rng, 3, 2048)
        first, last = rng.randint(0, 1), rng.randint(1, 2)
        keep = rng.randint(first + last, max(first + last, pages))
        return _evict(B, pages, keep, first, last, mix)
    if kind == "append":
        start = 64 * rng.randint(0, 40)
        hi = _log_int(rng, 1, 16384)
        B = _log_int(rng, 1, max(1, min(64, 32768 * 1024 // (hi * Hkv * d))))
        return _append(B, Hkv, d, rng.randint(1, hi), hi, start, dtype, rng.random() < 0.5, mix)
    hi = _log_int(rng, 1, 32768)
    lo = rng.randint(1, hi)
    room = 64 * 16384 * 8 * 128 // (hi * Hkv * d)              # keys and values of the largest listed cache
    if kind == "attention":
        N = _log_int(rng, 2, 2048)
        room = min(room, 4 * 32 * 1024 * 8192 * 128 // (Hq * N * hi * d))
        while room < 1:
            N, hi = max(2, N // 2), max(1, hi // 2)
            lo = min(lo, hi)
            room = min(64 * 16384 * 8 * 128 // (hi * Hkv * d), 4 * 32 * 1024 * 8192 * 128 // (Hq * N * hi * d))
        B = _log_int(rng, 1, min(32, room))
        return _attention(B, Hq, Hkv, d, N, lo, hi, rng.random() < 0.5, dtype, mix)
    B = _log_int(rng, 1, max(1, min(64, room)))
    if kind == "step":
        return _step(B, Hq, Hkv, d, lo, hi, dtype, mix)
    return _decode(B, Hq, Hkv, d, lo, hi, dtype, rng.random() < 0.5, rng.random() < 0.5, mix)


def _lens(case):
    """Lengths of the sequences (tokens appended, for "append"): the longest first, the rest spread over the logarithm."""
    rng = random.Random(1000003 * case["mix"] + case["B"])
    return [case["hi"]] + [_log_int(rng, case["lo"], case["hi"]) for _ in range(case["B"] - 1)]


def _pages_of(n):
    return (n + 63) // 64


# ------------------------------------------------------------------ the format, in plain operations
def _scales(device, dtype=torch.float32):
    """The 256 values of a group's scale, S = 2^(e-48) (1 + M/4), ascending."""
    c = torch.arange(256, device=device)
    return torch.ldexp((4 + c % 4).to(dtype), (torch.div(c, 4, rounding_mode="floor") - 50).to(dtype))


def _quantize(x):
    """x [..., 64] FP32 -> signed codes [..., 64], shifts [..., 16], scale codes [...]."""
    S_all = _scales(x.device)
    A = x.abs().amax(-1)
    code = torch.searchsorted(7 * S_all, A.contiguous()).clamp(max=255)
    S = S_all[code]
    a = x.abs().unflatten(-1, (8, 2, 4)).amax(-1)
    need = (a > 1.75 * S[..., None, None]).int() + (a > 3.5 * S[..., None, None]).int()
    k = torch.maximum(need, (need.sum(-1, keepdim=True) >= 2).int()).flatten(-2)
    step = (S / 4)[..., None] * (1 << k).float()
    m = torch.round(x.unflatten(-1, (16, 4)) / step[..., None]).clamp(-7, 7).flatten(-2)
    return m.int(), k, code


def _bytes_of(words):
    """[..., n] integers below 2^32 -> [..., 4 n] bytes, least significant first."""
    return torch.stack([(words >> (8 * j)) & 255 for j in range(4)], -1).flatten(-2).to(torch.uint8)


def _nibble_words(c):
    w = c[..., 0].long()
    for e in range(1, 8):
        w = w | (c[..., e].long() << (4 * e))
    return w


def _pack_k(x):
    """Smoothed keys [..., 64, d] FP32 -> (codes, shifts, scales) as bytes, [..., 64, *]."""
    G = x.shape[-1] // 64
    m, k, code = _quantize(x.unflatten(-1, (G, 64)))
    w = _nibble_words((m + 8).unflatten(-1, (8, 8)))                             # [..., 64, G, 8]
    w = w.unflatten(-1, (4, 2)).movedim(-3, -2).flatten(-3)                      # [..., 64, 4 * G * 2]
    s = torch.zeros(k.shape[:-1], dtype=torch.long, device=x.device)
    for t in range(16):
        s = s | (k[..., t].long() << (16 * (t % 2) + 2 * (t // 2)))
    return _bytes_of(w), _bytes_of(s), code.to(torch.uint8)


def _pack_v(x):
    """Values [..., 64, d] FP32 -> (codes, shifts, scales) as bytes, [..., d, *]."""
    m, k, code = _quantize(x.transpose(-1, -2))
    c = (m + 8).unflatten(-1, (4, 2, 2, 4))                                      # token 16 i + 8 r + 4 h + e
    w = _nibble_words(c.transpose(-2, -3).flatten(-2)).flatten(-2)               # [..., d, i, h] of nibbles (r, e)
    k = k.unflatten(-1, (4, 2, 2))
    s = torch.zeros(code.shape, dtype=torch.long, device=x.device)
    for i in range(4):
        for r in range(2):
            for h in range(2):
                s = s | (k[..., i, r, h].long() << (16 * r + 2 * (2 * i + h)))
    return _bytes_of(w), _bytes_of(s[..., None]), code.to(torch.uint8)


def _regions(d):
    """Byte offsets of a head's part of a page: codes, shifts and scales of K, then of V."""
    off = [0]
    for n in (32 * d, 4 * d, d, 32 * d, 4 * d, d):
        off.append(off[-1] + n)
    return off


def _pack(k, v):
    """[..., 64, d] each -> pages [..., 74 d]."""
    kc, ks, ke = _pack_k(k)
    vc, vs, ve = _pack_v(v)
    return torch.cat([t.flatten(-2) for t in (kc, ks, ke, vc, vs)] + [ve], -1)


def _unpack(pages):
    """Pages [..., 74 d] -> the values they stand for, K and V [..., 64, d] FP32."""
    d = pages.shape[-1] // 74
    G, dev, o = d // 64, pages.device, _regions(d)
    part = [pages[..., o[i]:o[i + 1]] for i in range(6)]
    S = _scales(dev) / 4
    nib = torch.tensor([0, 4], dtype=torch.uint8, device=dev)

    def codes(b):
        return ((b[..., None] >> nib) & 15).flatten(-2).to(torch.int8) - 8       # in nibble order

    def shifts(b, t_of):
        w = b.unflatten(-1, (-1, 4)).int()
        return torch.stack([(w[..., t // 8] >> (t % 8)) & 3 for t in t_of], -1)

    lead = pages.shape[:-1]
    kc = codes(part[0]).reshape(lead + (64, 4, G, 2, 8)).movedim(-3, -4).reshape(lead + (64, G, 16, 4))
    ks = shifts(part[1], [16 * (t % 2) + 2 * (t // 2) for t in range(16)]).reshape(lead + (64, G, 16))
    ke = S[part[2].reshape(lead + (64, G)).int()]
    K = (kc.float() * ((1 << ks).float() * ke[..., None])[..., None]).reshape(lead + (64, d))
    vc = codes(part[3]).reshape(lead + (d, 4, 2, 2, 4)).transpose(-2, -3).reshape(lead + (d, 16, 4))
    vs = shifts(part[4], [16 * r + 2 * (2 * i + h) for i in range(4) for r in range(2) for h in range(2)])
    ve = S[part[5].int()]
    V = (vc.float() * ((1 << vs.reshape(lead + (d, 16))).float() * ve[..., None])[..., None]).reshape(lead + (d, 64))
    return K, V.transpose(-1, -2)


# ------------------------------------------------------------------ inputs
def _randn(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _factors(gen, Hkv, d, smooth):
    """Smooth-QK factors of keys with four outlier channels per head, and the gain of those channels."""
    gain = torch.ones(Hkv, d, device="cuda")
    if smooth:
        ch = torch.rand((Hkv, d), generator=gen, device="cuda").argsort(-1)[:, :4]
        gain.scatter_(1, ch, 20.0)
    s = gain.sqrt() * (1 + 0.1 * torch.rand((Hkv, d), generator=gen, device="cuda"))
    return gain, s


def _cache_pages(gen, n_pages, Hkv, d, dtype, gain, s):
    """Pages of quantized random keys and values: a pool of distinct ones, dealt out at random."""
    pool = max(4, min(64, n_pages))
    k = (_randn(gen, (pool, Hkv, 64, d), dtype) * gain[:, None]).to(dtype)
    k = (k.float() / s[:, None]).to(dtype)
    pages = _pack(k.float(), _randn(gen, (pool, Hkv, 64, d), dtype).float())
    pick = torch.randint(0, pool, (n_pages, Hkv), generator=gen, device="cuda")
    return pages[pick, torch.arange(Hkv, device="cuda")].contiguous()


def _table(gen, lens, spare):
    """Block table of sequences of these lengths: physical pages in random order, -1 behind the last."""
    need = [_pages_of(n) for n in lens]
    n_pages = sum(need) + spare
    perm = torch.rand(n_pages, generator=gen, device="cuda").argsort().int()
    table = torch.full((len(lens), max(need) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, n_pages


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case=case)
    if case["kind"] == "evict":
        B, P = case["B"], case["pages"]
        rng = random.Random(1000003 * case["mix"] + B)
        st["lens"] = [64 * P - 13] + [_log_int(rng, 1, 64 * P) for _ in range(B - 1)]
        st["kv_lens"] = _ints(st["lens"])
        st["table"], _ = _table(gen, st["lens"], 0)
        st["table"] = st["table"][:, :P].contiguous()
        # attention weight falls off over the pages' ranks, in random order; many pages got none at all
        w = torch.rand((B, P), generator=gen, device="cuda")
        st["weight"] = torch.where(w < 0.2, 0.0, 0.01 / (1.001 - w))
        if own:
            from paper_2607_04302_b200 import binding as hb
            st["out"] = hb.alloc_evicted(st["table"])
        return st
    Hkv, d, dt = case["Hkv"], case["d"], _DT[case["dtype"]]
    n = _lens(case)
    gain, s = _factors(gen, Hkv, d, case.get("smooth", True))
    st["s"], st["inv_s"] = s, 1.0 / s
    if case["kind"] == "append":
        start = [case["start"] if b % 2 == 0 else 0 for b in range(case["B"])]
        st["n_new"], st["starts"], st["lens"] = n, start, [a + b for a, b in zip(start, n)]
    else:
        st["lens"] = n
    B = case["B"]
    st["kv_lens"] = _ints(st["lens"])
    st["table"], n_pages = _table(gen, st["lens"], 3)
    if case["kind"] == "append":
        st["pages"] = torch.zeros((n_pages, Hkv, 74 * d), dtype=torch.uint8, device="cuda")
    else:
        st["pages"] = _cache_pages(gen, n_pages, Hkv, d, dt, gain, s)
    if case["kind"] in ("append", "step"):
        N = max(n) if case["kind"] == "append" else 1
        st["k"] = (_randn(gen, (B, Hkv, N, d), dt) * gain[:, None]).to(dt)
        st["v"] = _randn(gen, (B, Hkv, N, d), dt)
        st["v_tail"] = _randn(gen, (B, Hkv, 64, d), dt)
        if case["kind"] == "append":
            st["n_new_d"], st["start_d"] = _ints(n), _ints(st["starts"])
            st["read"] = [torch.zeros((B, Hkv, N, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        else:
            st["n_new"], st["starts"] = [1] * B, [x - 1 for x in n]
    else:
        st["v_tail"] = None
    if case["kind"] != "append":
        N = case.get("N", 1)
        # some heads look at few keys, some at many
        sharp = 0.5 + 2.5 * torch.rand((case["Hq"], 1, 1), generator=gen, device="cuda")
        st["q"] = (_randn(gen, (B, case["Hq"], N, d), torch.float32) * sharp).to(dt)
        if case["kind"] in ("step", "decode"):
            st["q"] = st["q"][:, :, 0].contiguous()
        if case["kind"] == "step" or case.get("weight"):
            st["weight"] = torch.rand(st["table"].shape, generator=gen, device="cuda")
            st["weight_out"] = torch.zeros_like(st["weight"])
    if own:
        from paper_2607_04302_b200 import binding as hb
        st["cache"] = hb.PagedCache(st["pages"], st["v_tail"])
    return st


# ------------------------------------------------------------------ plain forms
def _plain_append(st):
    c = st["case"]
    dt = _DT[c["dtype"]]
    for b, (n, start) in enumerate(zip(st["n_new"], st["starts"])):
        end, p0 = start + n, start // 64
        p1 = _pages_of(end)
        head = start - 64 * p0
        k = st["k"][b, :, :n]
        k = (k.float() * st["inv_s"][:, None]).to(dt).float() if c.get("smooth", True) else k.float()
        ids = st["table"][b, p0:p1].long()
        Hkv, d = k.shape[0], k.shape[-1]
        o, G = _regions(d), d // 64
        kc, ks, ke = _pack_k(k)
        t = torch.arange(head, head + n, device=k.device)
        pg, row = ids[t // 64], t % 64
        rows = st["pages"]
        for part, lo, width in ((kc, o[0], d // 2), (ks, o[1], 4 * G), (ke, o[2], G)):
            view = rows[:, :, lo:lo + 64 * width].unflatten(-1, (64, width))
            view[pg, :, row] = part.transpose(0, 1)
        v = torch.zeros((Hkv, 64 * (p1 - p0), d), device=k.device)
        v[:, :head] = st["v_tail"][b, :, :head].float()
        v[:, head:head + n] = st["v"][b, :, :n].float()
        vc, vs, ve = _pack_v(v.unflatten(1, (p1 - p0, 64)))
        for part, lo in ((vc, o[3]), (vs, o[4]), (ve[..., None], o[5])):
            flat = part.flatten(-2)
            rows[ids, :, lo:lo + flat.shape[-1]] = flat.transpose(0, 1)
        left = end % 64
        if left:
            st["v_tail"][b, :, :left] = v[:, 64 * (p1 - p0 - 1):64 * (p1 - p0 - 1) + left].to(dt)


def _plain_values(st, b, n):
    """K and V of the first n tokens of sequence b, [Hkv, n, d] FP32."""
    K, V = _unpack(st["pages"][st["table"][b, :_pages_of(n)].long()])
    return K.transpose(0, 1).flatten(1, 2)[:, :n], V.transpose(0, 1).flatten(1, 2)[:, :n]


def _plain_read(st):
    k_out, v_out = st["read"]
    for b, (n, start) in enumerate(zip(st["n_new"], st["starts"])):
        K, V = _plain_values(st, b, start + n)
        k_out[b, :, :n] = K[:, start:]
        v_out[b, :, :n] = V[:, start:]
    return {"k": k_out, "v": v_out, "v_tail": st["v_tail"]}


def _plain_attend(st):
    """Outputs, logarithms of the softmax sums and page weights of q [B, Hq, N, d] over the cache."""
    c = st["case"]
    dt, rep, d = _DT[c["dtype"]], c["Hq"] // c["Hkv"], c["d"]
    q = st["q"] if st["q"].dim() == 4 else st["q"][:, :, None]
    N = q.shape[2]
    s = st["s"].repeat_interleave(rep, 0)[:, None]
    out, lse = torch.zeros_like(q), torch.full(q.shape[:3], -math.inf, device=q.device)
    for b, n in enumerate(st["lens"]):
        K, V = _plain_values(st, b, n)
        for g in range(c["Hkv"]):
            hs = slice(g * rep, (g + 1) * rep)
            S = ((q[b, hs].float() * s[hs]).to(dt).float() @ K[g].T) / math.sqrt(d)
            if c.get("causal"):
                pos = n - N + torch.arange(N, device=q.device)
                seen = torch.arange(n, device=q.device)[None] <= pos[:, None]
                S = S.masked_fill(~seen, -math.inf)
            m = S.amax(-1, keepdim=True)
            m = torch.where(m == -math.inf, torch.zeros_like(m), m)
            P = torch.exp(S - m)
            l = P.sum(-1, keepdim=True)
            out[b, hs] = (P @ V[g] / torch.where(l == 0, torch.ones_like(l), l)).to(dt)
            lse[b, hs] = (m + torch.log(l))[..., 0]
            if "weight" in st:
                p = P[:, 0] / l[:, 0]
                np_ = _pages_of(n)
                per = torch.nn.functional.pad(p, (0, 64 * np_ - n)).unflatten(-1, (np_, 64)).sum(-1).sum(0)
                if g == 0:
                    st["weight_out"][b, :np_] = st["weight"][b, :np_]
                st["weight_out"][b, :np_] += per
    return out, lse


def _plain_evict(st):
    c, table, w = st["case"], st["table"], st["weight"]
    B, P = table.shape
    idx = torch.arange(P, device=table.device)[None]
    np_ = ((st["kv_lens"] + 63) // 64)[:, None]
    fixed = (idx < c["first"]) | ((idx >= np_ - c["last"]) & (idx < np_))
    key = torch.where(fixed, math.inf, w).masked_fill(idx >= np_, -math.inf)
    order = key.argsort(dim=1, descending=True, stable=True)
    rank = torch.empty_like(order).scatter_(1, order, idx.expand(B, P).contiguous())
    keep = (rank < c["keep"]) & (idx < np_)
    gone = ~keep & (idx < np_)

    def compact(mask, values, fill):
        pos = torch.where(mask, mask.cumsum(1) - 1, P)                            # slot P collects what is not taken
        out = torch.full((B, P + 1), fill, dtype=values.dtype, device=values.device)
        return out.scatter_(1, pos, values)[:, :P].contiguous()

    n_gone = gone.sum(1, dtype=torch.int32)
    return {"table": compact(keep, table, -1), "kv_lens": st["kv_lens"] - 64 * n_gone,
            "weight": compact(keep, w, 0.0), "freed": compact(gone, table, -1), "n_freed": n_gone}


def run(state):
    st, c = state, state["case"]
    kind = c["kind"]
    if own:
        from paper_2607_04302_b200 import binding as hb
        if kind == "evict":
            r = hb.cache_evict(st["table"], st["kv_lens"], st["weight"], c["keep"], c["first"], c["last"], out=st["out"])
            return {"table": r.block_table, "kv_lens": r.kv_lens, "weight": r.page_weight, "freed": r.freed,
                    "n_freed": r.n_freed}
        if kind == "append":
            hb.cache_append(st["cache"], st["k"], st["v"], st["table"], st["kv_lens"], n_new=st["n_new_d"],
                            inv_s=st["inv_s"] if c["smooth"] else None)
            k, v = hb.cache_read(st["cache"], st["table"], st["kv_lens"], st["k"].shape[2], start=st["start_d"],
                                 out=st["read"])
            return {"k": k, "v": v, "v_tail": st["v_tail"]}
        if kind == "attention":
            return {"out": hb.cache_attention(st["q"], st["cache"], st["table"], st["kv_lens"], c["causal"], s=st["s"])}
        if kind == "step":
            hb.cache_append(st["cache"], st["k"], st["v"], st["table"], st["kv_lens"], inv_s=st["inv_s"])
        r = {}
        lse = torch.empty(st["q"].shape[:2], device=st["q"].device) if c.get("lse") else None
        r["out"] = hb.cache_decode(st["q"], st["cache"], st["table"], st["kv_lens"], s=st["s"], lse=lse,
                                   page_weight=st.get("weight"), page_weight_out=st.get("weight_out"))
        if lse is not None:
            r["lse"] = lse
    else:
        if kind == "evict":
            return _plain_evict(st)
        if kind == "append":
            _plain_append(st)
            return _plain_read(st)
        if kind == "step":
            _plain_append(st)
        out, lse = _plain_attend(st)
        if kind == "attention":
            return {"out": out}
        r = {"out": out[:, :, 0]}
        if c.get("lse"):
            r["lse"] = lse[:, :, 0]
    if "weight_out" in st:
        r["weight"] = st["weight_out"]
    if kind == "step":
        r["v_tail"] = st["v_tail"]
    return r


def work(case):
    if case["kind"] == "evict":
        n = case["B"] * case["pages"]
        return {"bytes": 4 * (2 * n + 3 * n + 3 * case["B"]), "flops": n}
    B, Hkv, d = case["B"], case["Hkv"], case["d"]
    tok = sum(_lens(case)) * Hkv * d                              # elements of K, and of V
    packed = 2 * tok * 4.5 / 8
    if case["kind"] == "append":
        return {"bytes": 2 * tok * 2 + 2 * packed + 2 * tok * 2, "flops": 2 * tok * 4}
    N, Hq = case.get("N", 1), case["Hq"]
    pairs = sum(_lens(case)) * N
    if case.get("causal"):
        pairs = sum(sum(max(0, n - N + 1 + i) for i in range(N)) for n in _lens(case))
    b = packed + 2 * 2 * B * Hq * N * d + 4 * Hkv * d
    if case["kind"] == "step":
        b += 4 * B * Hkv * d + 2 * sum((n - 1) % 64 + 1 for n in _lens(case)) * Hkv * d
    if case["kind"] == "step" or case.get("weight"):
        b += 8 * sum(_pages_of(n) for n in _lens(case))
    return {"bytes": b, "flops": 4 * pairs * Hq * d}


# ------------------------------------------------------------------ the definition in 64 bits
_TABLE64 = [(4 + c % 4) * 2.0 ** (c // 4 - 50) for c in range(256)]


def _hif4_64(x):
    """HIF4 values of groups x [..., 64] (FP64): smallest scale with 7 S >= max, least shift that holds each subgroup."""
    S_all = torch.tensor(_TABLE64, dtype=torch.float64, device=x.device)
    top = x.abs().max(-1, keepdim=True).values
    S = S_all[(top > 7 * S_all).sum(-1).clamp(max=255)].unsqueeze(-1).unsqueeze(-1)
    x8 = x.reshape(x.shape[:-1] + (8, 8))
    lo, hi = x8[..., :4].abs().amax(-1, keepdim=True), x8[..., 4:].abs().amax(-1, keepdim=True)

    def exceeded(a):
        return (a > 1.75 * S).double() + (a > 3.5 * S).double()

    n_lo, n_hi = exceeded(lo), exceeded(hi)
    both = ((n_lo == 2) | (n_hi == 2) | ((n_lo >= 1) & (n_hi >= 1))).double()
    k = torch.cat([torch.maximum(n_lo, both).expand(x8.shape[:-1] + (4,)),
                   torch.maximum(n_hi, both).expand(x8.shape[:-1] + (4,))], -1)
    step = S / 4 * 2.0 ** k
    return (torch.round(x8 / step).clamp(-7, 7) * step).reshape(x.shape)


def _values_64(pages):
    """K and V of heads' parts of pages [n, 74 d] in FP64, from 32-bit words."""
    n, d = pages.shape[0], pages.shape[1] // 74
    G, dev = d // 64, pages.device
    S = torch.tensor(_TABLE64, dtype=torch.float64, device=dev) / 4
    k_half, v_half = pages[:, :37 * d], pages[:, 37 * d:]
    kw, vw = (t[:, :36 * d].contiguous().view(torch.int32).long() & 0xFFFFFFFF for t in (k_half, v_half))
    kw, kx, vw, vx = kw[:, :8 * d], kw[:, 8 * d:], vw[:, :8 * d], vw[:, 8 * d:]
    K = torch.empty((n, 64, d), dtype=torch.float64, device=dev)
    kw, kx = kw.reshape(n, 64, 8 * G), kx.reshape(n, 64, G)
    ks = S[k_half[:, 36 * d:].long().reshape(n, 64, G)]
    for c in range(d):
        g, u, e = c // 64, c % 64 // 8, c % 8
        code = (kw[:, :, (u // 2) * 2 * G + 2 * g + u % 2] >> (4 * e)) % 16 - 8
        shift = (kx[:, :, g] >> (2 * u + 16 * (e // 4))) % 4
        K[:, :, c] = code * 2.0 ** shift * ks[:, :, g]
    V = torch.empty((n, 64, d), dtype=torch.float64, device=dev)
    vw, vs = vw.reshape(n, d, 8), S[v_half[:, 36 * d:].long()]
    for t in range(64):
        i, r, h, e = t // 16, t // 8 % 2, t // 4 % 2, t % 4
        code = (vw[:, :, 2 * i + h] >> (16 * r + 4 * e)) % 16 - 8
        shift = (vx >> (16 * r + 2 * (2 * i + h))) % 4
        V[:, t] = code * 2.0 ** shift * vs
    return K, V


def _exact_evict(case, seed):
    """The definition, one sequence after the other on the host: sort the middle pages by (weight falling, index rising)."""
    st = prepare(case, seed)
    table, weight = st["table"].cpu().numpy(), st["weight"].double().cpu().numpy()
    new_table, freed, new_weight = np.full_like(table, -1), np.full_like(table, -1), np.zeros_like(weight)
    lens, counts = [], []
    for b, n in enumerate(st["lens"]):
        pages = list(range(_pages_of(n)))
        gone = []
        if len(pages) > case["keep"]:
            middle = pages[case["first"]:len(pages) - case["last"]]
            middle.sort(key=lambda j: (-weight[b, j], j))
            gone = sorted(middle[case["keep"] - case["first"] - case["last"]:])
        left = sorted(set(pages) - set(gone))
        new_table[b, :len(left)], freed[b, :len(gone)] = table[b, left], table[b, gone]
        new_weight[b, :len(left)] = weight[b, left]
        lens.append(n - 64 * len(gone))
        counts.append(len(gone))
    return {"table": torch.from_numpy(new_table).cuda(), "kv_lens": _ints(lens),
            "weight": torch.from_numpy(new_weight).cuda(), "freed": torch.from_numpy(freed).cuda(), "n_freed": _ints(counts)}


def exact(case, seed):
    if case["kind"] == "evict":
        return _exact_evict(case, seed)
    Hkv, d, B = case["Hkv"], case["d"], case["B"]
    if case["kind"] != "append" and (sum(_lens(case)) * d * case.get("N", 1) * case["Hq"] > 1 << 39 or B * case["Hq"] > 4096):
        return None
    st = prepare(case, seed)
    dt = _DT[case["dtype"]]
    smooth = case.get("smooth", True)

    def smoothed(x, f):                                       # one FP32 product, rounded to the type of x
        return (x.double() * f.double()).float().to(dt).double() if smooth else x.double()

    if case["kind"] == "append":
        k_out, v_out = (t.double() for t in st["read"])
        tail = st["v_tail"].double()
        for b, (n, start) in enumerate(zip(st["n_new"], st["starts"])):
            for g in range(Hkv):
                k = smoothed(st["k"][b, g, :n], st["inv_s"][g])
                k_out[b, g, :n] = _hif4_64(k.reshape(n, d // 64, 64)).reshape(n, d)
                v = torch.zeros((_pages_of(n), 64, d), dtype=torch.float64, device=k.device)
                v.view(-1, d)[:n] = st["v"][b, g, :n].double()           # the chunk starts a page
                v_out[b, g, :n] = _hif4_64(v.transpose(1, 2)).transpose(1, 2).reshape(-1, d)[:n]
                if n % 64:
                    tail[b, g, :n % 64] = v[-1, :n % 64]
        return {"k": k_out, "v": v_out, "v_tail": tail}
    rep = case["Hq"] // Hkv
    q = st["q"].reshape(B, case["Hq"], -1, d)
    N = q.shape[2]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device=q.device)
    weight = st["weight_out"].double() if "weight" in st else None
    for b, n in enumerate(st["lens"]):
        np_ = _pages_of(n)
        if weight is not None:
            weight[b, :np_] = st["weight"][b, :np_].double()
        K_all, V_all = (t.unflatten(0, (np_, Hkv)) for t in _values_64(st["pages"][st["table"][b, :np_].long()].flatten(0, 1)))
        for g in range(Hkv):
            K, V = K_all[:, g].clone(), V_all[:, g].clone()
            if case["kind"] == "step":
                r = (n - 1) % 64
                K[-1, r] = _hif4_64(smoothed(st["k"][b, g, 0], st["inv_s"][g]).reshape(-1, 64)).reshape(-1)
                v = torch.zeros((64, d), dtype=torch.float64, device=q.device)
                v[:r] = st["v_tail"][b, g, :r].double()
                v[r] = st["v"][b, g, 0].double()
                V[-1] = _hif4_64(v.T).T
            K, V = K.reshape(-1, d)[:n], V.reshape(-1, d)[:n]
            for h in range(g * rep, (g + 1) * rep):
                S = smoothed(q[b, h], st["s"][g]) @ K.T / math.sqrt(d)
                if case.get("causal"):
                    row = torch.arange(N, device=q.device)[:, None]
                    S[torch.arange(n, device=q.device)[None] > row + (n - N)] = -math.inf
                lse[b, h] = torch.logsumexp(S, -1)
                P = torch.exp(S - torch.where(lse[b, h] == -math.inf, 0.0, lse[b, h])[:, None])
                out[b, h] = P @ V
                if weight is not None:
                    for_page = torch.zeros(64 * np_, dtype=torch.float64, device=q.device)
                    for_page[:n] = P[0]
                    weight[b, :np_] += for_page.view(np_, 64).sum(-1)
    if case["kind"] == "attention":
        return {"out": out}
    r = {"out": out[:, :, 0]}
    if case.get("lse"):
        r["lse"] = lse[:, :, 0]
    if weight is not None:
        r["weight"] = weight
    if case["kind"] == "step":
        tail = st["v_tail"].double()
        for b, n in enumerate(st["lens"]):
            if n % 64:
                tail[b, :, n % 64 - 1] = st["v"][b, :, 0].double()
        r["v_tail"] = tail
    return r
