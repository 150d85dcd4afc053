"""Paged HIF4 cache, restated for the tests: page bytes from the oracle's codes and metadata, values of pages and attention over
them in FP64, eviction by sorting.  Shares no code with the kernels."""
import math
from types import SimpleNamespace

import numpy as np
import torch

from oracle import hifa4_oracle as orc

_S4 = np.array([(4 + c % 4) * 2.0 ** (c // 4 - 52) for c in range(256)])     # S / 4


def _signed(nib):
    return np.where(nib & 8, -(nib & 7).astype(np.int64), (nib & 7).astype(np.int64))


def quantize_groups(x):
    """x [..., 64] FP64 -> signed codes [..., 64], shifts [..., 16], scale codes [...] of the oracle's quantizer."""
    shape = x.shape[:-1]
    r = orc.hif4_quantize_rows(np.ascontiguousarray(x.reshape(-1, 64), dtype=np.float64))
    codes = np.stack([r[0] & 15, r[0] >> 4], -1).reshape(-1, 64)             # even element in the low nibble
    meta = r[1].reshape(-1).astype(np.int64)
    t = np.arange(16)
    shifts = ((meta[:, None] >> (8 + t // 2)) & 1) + ((meta[:, None] >> (16 + t)) & 1)
    return _signed(codes).reshape(shape + (64,)), shifts.reshape(shape + (16,)), (meta & 255).reshape(shape)


def page_bytes(k, v):
    """Smoothed keys and values [64, d] FP64 -> the 74 d bytes of a head's part of a page."""
    d = k.shape[1]
    G = d // 64
    out = []
    for x, is_v in ((k, False), (v, True)):
        rows = x.T if is_v else x
        m, sh, code = quantize_groups(rows.reshape(-1, 64))
        words, shifts = np.zeros((len(m), 8), np.uint64), np.zeros(len(m), np.uint64)
        for e in range(64):
            if is_v:                                     # token e
                i, r, h, n = e // 16, e // 8 % 2, e // 4 % 2, e % 4
                w, nib = 2 * i + h, 4 * r + n
            else:
                w, nib = e // 8, e % 8
            words[:, w] |= (m[:, e] + 8).astype(np.uint64) << np.uint64(4 * nib)
        for t in range(16):
            if is_v:
                i, r, h = t // 4, t // 2 % 2, t % 2
                bit = 16 * r + 2 * (2 * i + h)
            else:
                bit = 16 * (t % 2) + 2 * (t // 2)
            shifts |= sh[:, t].astype(np.uint64) << np.uint64(bit)
        if not is_v:                                     # [64][G][p][2] -> [64][p][G][2]
            words = words.reshape(64, G, 4, 2).transpose(0, 2, 1, 3)
        out += [words.astype("<u4").tobytes(), shifts.astype("<u4").tobytes(), code.astype(np.uint8).tobytes()]
    return np.frombuffer(b"".join(out), np.uint8)


def values(page):
    """A head's part of a page [74 d] -> K, V [64, d] FP64."""
    page = np.asarray(page)
    d = page.size // 74
    G, half = d // 64, 37 * d
    res = []
    for is_v in (False, True):
        part = page[half:] if is_v else page[:half]
        words = np.frombuffer(part[:32 * d].tobytes(), "<u4").astype(np.int64)
        shifts = np.frombuffer(part[32 * d:36 * d].tobytes(), "<u4").astype(np.int64)
        scale = _S4[part[36 * d:37 * d]]
        words = words.reshape(d, 8) if is_v else words.reshape(64, 4, G, 2).transpose(0, 2, 1, 3).reshape(64 * G, 8)
        x = np.zeros((len(words), 64))
        for e in range(64):
            if is_v:
                i, r, h, n = e // 16, e // 8 % 2, e // 4 % 2, e % 4
                w, nib, bit = 2 * i + h, 4 * r + n, 16 * r + 2 * (2 * i + h)
            else:
                w, nib, bit = e // 8, e % 8, 16 * (e // 4 % 2) + 2 * (e // 8)
            x[:, e] = (((words[:, w] >> (4 * nib)) & 15) - 8) * 2.0 ** ((shifts >> bit) & 3) * scale
        res.append(x.T if is_v else x.reshape(64, d))
    return res


def round_in(x, dtype):
    """FP64 -> nearest FP32 -> nearest value of the activation dtype, as FP64."""
    return x.float().to(dtype).double()


def sequence(pages, table_row, n, h):
    """K, V [n, d] FP64 (CPU) of one sequence's head h; pages: uint8 CPU tensor."""
    ks, vs = [], []
    for j in range((n + 63) // 64):
        k, v = values(pages[int(table_row[j]), h].numpy())
        ks.append(k)
        vs.append(v)
    if not ks:
        d = pages.shape[-1] // 74
        return torch.zeros(0, d, dtype=torch.float64), torch.zeros(0, d, dtype=torch.float64)
    return torch.from_numpy(np.concatenate(ks))[:n], torch.from_numpy(np.concatenate(vs))[:n]


def attend(q, pages, table, lens, s=None, causal=False, q_to_kv=None, scale=None):
    """q [B,Hq,N,d] (CPU, 16-bit), everything on the CPU, FP64.  Returns out, lse [B,Hq,N], page weights [B,max_pages] (summed
    over heads and queries) and three bounds: A = sum_j p_j |v_j| and W = sum_j |v_j| [B,Hq,N,d], E = max_j sum_c |q_c k_jc| * scale
    [B,Hq,N]."""
    B, Hq, N, d = q.shape
    Hkv = pages.shape[1]
    scale = scale or 1 / math.sqrt(d)
    q_to_kv = q_to_kv or [h // (Hq // Hkv) for h in range(Hq)]
    out, A, W = (torch.zeros(q.shape, dtype=torch.float64) for _ in range(3))
    lse = torch.full((B, Hq, N), -math.inf, dtype=torch.float64)
    E = torch.zeros((B, Hq, N), dtype=torch.float64)
    weight = torch.zeros(table.shape, dtype=torch.float64)
    for b in range(B):
        n = int(lens[b])
        kv = {}
        for h in range(Hq):
            g = q_to_kv[h]
            if g not in kv:
                kv[g] = sequence(pages, table[b], n, g)
            K, V = kv[g]
            qq = q[b, h].double()
            if s is not None:
                qq = round_in(qq * s[g].double(), q.dtype)
            S = qq @ K.T * scale
            if causal:
                S = S.masked_fill(torch.arange(n)[None] > torch.arange(N)[:, None] + (n - N), -math.inf)
            if n:
                lse[b, h] = torch.logsumexp(S, -1)
                E[b, h] = (qq.abs() @ K.abs().T * scale).amax(-1)
            P = torch.where(S == -math.inf, 0.0, torch.exp(S - lse[b, h][:, None]))
            out[b, h], A[b, h], W[b, h] = P @ V, P @ V.abs(), (S > -math.inf).double() @ V.abs()
            per = torch.zeros(64 * ((n + 63) // 64), dtype=torch.float64)
            per[:n] = P.sum(0)
            weight[b, :(n + 63) // 64] += per.view(-1, 64).sum(-1)
    return SimpleNamespace(out=out, lse=lse, weight=weight, A=A, W=W, E=E)


def score_error(E, d):
    """Bound on the error of a score (natural units): FP32 sums of d products in any order, each step 2^-23 of the sum of magnitudes
    (tensor-core sums may be cut instead of rounded), the group scales and the factor in the exponent 2^-22 more."""
    return (d + 4) * 2.0 ** -23 * E


def tolerance(r, d, dtype, p_bits):
    """Bound on |kernel - exact| for the result r of attend: every p off by a factor 1 + eps (its rounding to p_bits, the
    exponential and the FP32 sums 2^-20, the score's error), in numerator and denominator.  FP16 numbers below 2^-14 have a
    spacing of 2^-24 whatever their size: with P = 2^15 at the row's maximum, where sum p >= 1, a p is off by half of 2^-24 2^-15 of
    that, 2^-40 per key, times |v|.  Then the rounding of the output, half a step of its type."""
    err = 2 * (2.0 ** -p_bits + 2.0 ** -20 + torch.expm1(score_error(r.E, d)))[..., None] * r.A + 2.0 ** -40 * r.W
    half = torch.finfo(dtype).eps / 2
    tiny = torch.finfo(dtype).smallest_normal * half                      # half a step below the smallest normal number
    return (r.out.abs() + err) * half + err + tiny


def evict(table, lens, weight, keep, first, last):
    """Plain Python; lists of rows, as cache_evict returns them."""
    B, P = table.shape
    res = dict(table=np.full((B, P), -1), lens=[], weight=np.zeros((B, P), np.float32), freed=np.full((B, P), -1), n=[])
    for b in range(B):
        np_ = (int(lens[b]) + 63) // 64
        gone = []
        if np_ > keep:
            mid = sorted(range(first, np_ - last),
                         key=lambda j: (math.isnan(weight[b, j]), 0.0 if math.isnan(weight[b, j]) else -float(weight[b, j]), j))
            gone = sorted(mid[keep - first - last:])
        left = [j for j in range(np_) if j not in set(gone)]
        res["table"][b, :len(left)] = table[b, left]
        res["weight"][b, :len(left)] = weight[b, left]
        res["freed"][b, :len(gone)] = table[b, gone]
        res["lens"].append(int(lens[b]) - 64 * len(gone))
        res["n"].append(len(gone))
    return res
