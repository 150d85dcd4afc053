"""Binding of the paged HIF4 cache without a GPU: import, and refusals by what the tensors say of themselves."""
import os
import subprocess
import sys

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
