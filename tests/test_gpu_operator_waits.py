"""The operators' bounded wait, on a barrier that nothing arrives at: it gives up, says so, and the device goes on.

The self-checking build has a kernel that does nothing else (a tenth of a second, by one warp)."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import ctypes as C, sys, time
import torch
sys.path.insert(0, sys.argv[1])
import paper_2609_39350_b200 as hap
L = hap.load_library()
assert hap.hap_operator_status() == 0
assert L.hap_operator_wait_check(C.c_uint64(1 << 40), C.c_void_p(0)) == 1
torch.cuda.synchronize()
began = time.monotonic()
assert L.hap_operator_wait_check(C.c_uint64(100_000_000), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
assert hap.hap_operator_status() == 1
assert 0.09 < time.monotonic() - began < 5
assert hap.hap_operator_status() == 0
x, w, off = torch.ones(200, 64, device="cuda", dtype=torch.bfloat16), torch.ones(1, 72, 64, device="cuda", dtype=torch.bfloat16), torch.tensor([0, 200], device="cuda")
assert (hap.hap_expert_matmul(x, w, off) == 64).all() and hap.hap_operator_status() == 0
print("DONE")
"""


def test_a_wait_that_runs_out_is_reported():
    from paper_2609_39350_b200.build import build_library
    build_library(checked=True)
    r = subprocess.run([sys.executable, "-c", CHILD, ROOT], env=dict(os.environ, HAP_LIBRARY="checked"), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "DONE" in r.stdout, r.stderr[-2000:]
