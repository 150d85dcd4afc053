"""Binding of the paged HIF4 cache without a GPU: import, and refusals by what the tensors say of themselves."""
import os
import subprocess
import sys
from types import SimpleNamespace

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_import_and_size_queries_on_a_torch_without_cuda():
    """Such a torch lacks the functions for the current device and stream."""
    code = ("import torch\n"
            "for n in ('_cuda_getDevice', '_cuda_getCurrentRawStream'):\n"
            "    if hasattr(torch._C, n): delattr(torch._C, n)\n"
            "from paper_2607_04302_b200 import binding as hb, build\n"
            "build.build()\n"
            "assert hb.cache_page_bytes(128) == 9472\n"
            "assert hb.quant_bytes(1, 32, 8, 4096, 128, hb.BF16, hb.Q, hb.CODES) > 0\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def _fake(shape, dtype, device):
    """What PagedCache asks of a tensor, on a device of this number (-1: the host)."""
    return SimpleNamespace(shape=torch.Size(shape), dtype=dtype, is_cuda=device >= 0, dim=lambda: len(shape), is_contiguous=lambda: True,
                           get_device=lambda: device, data_ptr=lambda: 256)


@pytest.mark.parametrize("pages_at,tail_at,ok", [(0, 0, True), (1, 1, True), (0, 1, False), (1, 0, False), (0, -1, False), (-1, -1, False)])
def test_pages_and_tails_are_on_one_device(pages_at, tail_at, ok):
    """A kernel takes both as pointers of its own device."""
    from paper_2607_04302_b200 import binding as hb
    pages, tail = _fake((4, 2, 74 * 64), torch.uint8, pages_at), _fake((3, 2, 64, 64), torch.float16, tail_at)
    if ok:
        hb.PagedCache(pages, tail)
    else:
        with pytest.raises(AssertionError):
            hb.PagedCache(pages, tail)


def test_outputs_that_overlap_the_queries_are_told():
    """A tensor over its own queries, or over a part of them; neighbours and interleaved views are fine."""
    from paper_2607_04302_b200 import binding as hb
    buf = torch.zeros(4, 6, 64, dtype=torch.float16)
    q, other = buf[:2], buf[2:]
    assert hb._apart(other, q) and hb._apart(q, other) and hb._apart(torch.zeros(2, 6, 64), q)
    assert not hb._apart(q, q) and not hb._apart(buf[1:3], q) and not hb._apart(q, buf[1:3]) and not hb._apart(buf, other)
    view = buf[:, 2:4]                                       # heads 2 and 3 of every row
    assert not hb._apart(buf, view) and hb._apart(torch.zeros(4, 2, 64), view) and hb._apart(buf[0, :2], view)
