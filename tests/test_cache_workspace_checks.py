"""What the join of the cache's decode kernel reads by numbers from the workspace (host build of the check, csrc/hifa4_cache.cuh): after a
decode that gave up they may be anything, and no number may lead it out of the workspace or into a long loop."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
CTAS = 148


@pytest.mark.skipif(not os.path.exists(NVCC), reason="needs nvcc")
def test_only_ranges_of_ctas_pass(tmp_path):
    src, so = tmp_path / "check.cu", tmp_path / "check.so"
    src.write_text('#include "hifa4_cache.cuh"\nextern "C" int check(int a, int b) { return hifa4::segment_recorded(a, b); }\n'
                   'extern "C" int ctas() { return hifa4::DECODE_CTAS; }\n')
    subprocess.run([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-shared", "-Xcompiler", "-fPIC",
                    "-I" + os.path.join(ROOT, "paper_2607_04302_b200", "csrc"), str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    assert lib.ctas() == CTAS
    rng = random.Random(0)
    ends = [0, 1, 2, 146, 147, 148, 149, -1, -2, -3, -5, 2 ** 31 - 1, -2 ** 31, 0x3F800000, -0x40800000]
    pairs = [(a, b) for a in ends for b in ends] + [(rng.randrange(-2 ** 31, 2 ** 31), rng.randrange(-2 ** 31, 2 ** 31)) for _ in range(1000)]
    for a, b in pairs:
        assert bool(lib.check(a, b)) == (0 <= a <= b < CTAS), (a, b)
