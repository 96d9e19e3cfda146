"""First calls of a process captured into a graph, and calls from two threads, for each variant of the attention's kernel
(its attributes are set once per instance): 7 query heads per KV head, and 20, whose rings are read by two warps; 10 per
KV head, one warp with two groups of 8 rows, is in test_gpu_paged."""

import os
import subprocess
import sys

import pytest

from test_gpu_paged import FIRST_CALLS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq", [28, 80])
def test_first_calls_of_every_variant(hq):
    heads = "n, hq, hkv = 300, 40, 4"
    assert heads in FIRST_CALLS
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    program = FIRST_CALLS.replace(heads, f"n, hq, hkv = 300, {hq}, 4")
    r = subprocess.run([sys.executable, "-c", program, root], capture_output=True, text=True, cwd=root, timeout=600)
    assert r.returncode == 0 and "first calls ok" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
