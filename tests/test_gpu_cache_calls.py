"""Calls of the paged HIF4 cache that its documentation allows, or that the binding has to refuse, beside those of test_gpu_cache.py."""
import math

import pytest
import torch

from tests import cache_reference as ref
from tests.test_gpu_cache import DEV, hb, ints, make_cache

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
