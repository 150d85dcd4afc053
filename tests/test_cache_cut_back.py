"""Sequences of the paged HIF4 cache that are cut back (drafted tokens taken back): which lengths hifa4_cache_append allows, checked
on a model of the rows that v_tail holds, and what the pages hold after appends behind such cuts, byte for byte."""
import random

import pytest
import torch

from tests import test_gpu_cache as gpu


def may_cut(begin, end, to):
    """The header's rule: the last append took the positions [begin, end); whether the sequence may be cut back to `to`."""
    last = (end - 1) // 64                                   # its last page
    return to % 64 == 0 or (to // 64 == last and (end % 64 != 0 or begin > 64 * last))


class Tail:
    """The positions whose raw values the rows of v_tail hold.  keep: whether an append that completes a page leaves rows."""

    def __init__(self, keep):
        self.rows, self.keep = [None] * 64, keep

    def append(self, begin, end, seq):
        """Tokens [begin, end) of the list seq (longer where the sequence is), which names every position's present token.
        Returns whether the rows that the first page is completed from are those of its present tokens."""
        first, last = begin // 64, (end - 1) // 64
        right = all(self.rows[r] == seq[64 * first + r] for r in range(begin % 64))
        t0 = begin % 64 if first == last else 0
        t1 = end % 64 or (63 if self.keep and t0 else 0)
        for r in range(t0, t1):
            self.rows[r] = seq[64 * last + r]
        return right


def run(begin, end, to, more, keep=True):
    """Appends [0, begin) and [begin, end), cuts back, appends `more` tokens."""
    tail, ok = Tail(keep), True
    seq = [("first", i) for i in range(end)]
    if begin:
        ok = tail.append(0, begin, seq)
    ok = tail.append(begin, end, seq) and ok
    assert ok                                                # without cuts the rows are always there
    seq = seq[:to] + [("second", i) for i in range(to, to + more)]
    return tail.append(to, to + more, seq)


LENGTHS = [0, 5, 60, 63, 64, 65, 127, 130]


def test_rows_are_there_wherever_the_rule_allows_a_cut():
    for begin in LENGTHS:
        for end in range(begin + 1, begin + 140):
            for to in range(0, end):
                if may_cut(begin, end, to):
                    assert run(begin, end, to, 1), (begin, end, to)


def test_rows_are_not_there_where_it_does_not():
    """The rule's bounds are needed, and so are the rows of a page that an append completes: 60 tokens and four drafted ones, of which
    two stay."""
    assert may_cut(60, 64, 62) and run(60, 64, 62, 1) and not run(60, 64, 62, 1, keep=False)
    assert not may_cut(0, 128, 100) and not run(0, 128, 100, 1)
    assert not may_cut(60, 70, 62) and not run(60, 70, 62, 1)
    assert not may_cut(60, 128, 100) and not run(60, 128, 100, 1)
    assert may_cut(63, 64, 63) and may_cut(60, 63, 61) and may_cut(60, 70, 66) and may_cut(60, 70, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("d,dtype", [(64, "fp16"), (128, "bf16"), (256, "bf16")])
def test_cut_back_and_appended_again(d, dtype):
    """Drafts that stay inside a page, complete one, and cross into the next, taken back in part: pages equal those of one append of the
    tokens that stayed.  Where the rule does not allow the cut, the page's tokens are appended again from its first position."""
    H, B, n = 2, 4, 250
    hb, dev, dt = gpu.hb(), gpu.DEV, gpu.DT[dtype]
    gen, rng = torch.Generator().manual_seed(d), random.Random(d)
    k, v = (torch.randn((B, H, n, d), generator=gen).to(dt) for _ in range(2))
    inv_s = (torch.rand((H, d), generator=gen) + 0.5).to(dev)
    cache = hb.alloc_cache(B * 4, H, d, dt, dev, B)
    cache.v_tail.normal_(generator=torch.Generator(dev).manual_seed(d))
    table = torch.randperm(B * 4, generator=gen).int().view(B, 4).to(dev).contiguous()

    def append(begin, end, kk, vv):
        """Positions [begin[b], end[b]) of each sequence."""
        new = [e - b for b, e in zip(begin, end)]
        part = [torch.zeros((B, H, max(new), d), dtype=dt) for _ in range(2)]
        for b in range(B):
            for x, src in zip(part, (kk, vv)):
                x[b, :, :new[b]] = src[b, :, begin[b]:end[b]]
        hb.cache_append(cache, part[0].to(dev), part[1].to(dev), table, gpu.ints(end), n_new=gpu.ints(new), inv_s=inv_s)

    kept = [60, 64, 1, 127]
    append([0] * B, kept, k, v)
    direct = again = full = 0
    while min(kept) < n - 12:
        # many drafts end where the page does
        drafts = [min(64 - x % 64 if x % 64 > 40 and rng.random() < 0.25 else rng.choice([1, 3, 7, 10, 20]), n - x) for x in kept]
        end = [x + y for x, y in zip(kept, drafts)]
        kd, vd = k.clone(), v.clone()                        # other tokens where the draft will be taken back
        to = [x + rng.randint(0, y) if y else x for x, y in zip(kept, drafts)]
        for b in range(B):
            kd[b, :, to[b]:], vd[b, :, to[b]:] = 3 * k[b, :, to[b]:].flip(1), -2 * v[b, :, to[b]:].flip(1)
        append(kept, end, kd, vd)
        begin = []
        for x, e, t in zip(kept, end, to):
            plain = e == x or t == e or may_cut(x, e, t)
            direct, again, full = direct + plain, again + (not plain), full + (e % 64 == 0 and x < t < e)
            begin.append(t if plain else t // 64 * 64)
        kept = [min(t + 1, n) for t in to]                   # the token that is sampled instead
        append(begin, kept, k, v)
        gpu.check_pages(cache, table.cpu(), k, v, inv_s, kept)
    assert direct > 20 and again > 1 and full > 2, (direct, again, full)
