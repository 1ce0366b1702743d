"""A host allocation that fails is a status, not an exception that ends the process (CPU, in a child process whose
address space is limited)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
COMMON = """
import ctypes as C, resource, sys
sys.path.insert(0, %r)
import numpy as np
from paper_2503_22562_amd import hb as H
lib = H.load()
class Shape:
    hidden, n_q_heads, n_kv_heads, head_dim, ffn_dim = 256, 4, 2, 64, 688
    rope_theta, rms_eps, kv_block = 5e5, 1e-5, 16
cfg = H.make_config(Shape, 1 << 20, 1 << 20)
def limit(extra):
    used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
    resource.setrlimit(resource.RLIMIT_AS, (used + extra, resource.RLIM_INFINITY))
"""
CALLS = {
    # marks for every block of a pool of 2^31 - 1
    "hb_validate_batch": """
reqs = [(5, 0, [3])]
limit(1 << 30)
status = H.hb_validate_batch(cfg, (1 << 31) - 1, reqs, 0x1000, 0x100000)
resource.setrlimit(resource.RLIMIT_AS, (resource.RLIM_INFINITY,) * 2)
assert H.hb_validate_batch(cfg, 4, reqs, 0x1000, 0x100000) == H.HB_OK
""",
    # where each of 2^31 - 1 blocks goes
    "hb_plan_compaction": """
src, n = np.zeros(4, np.int32), C.c_int32()
limit(1 << 30)
status = lib.hb_plan_compaction((1 << 31) - 1, None, None, 0, src.ctypes.data, src.ctypes.data, C.byref(n), C.byref(n))
""",
    # a batch of 2^26 decodes
    "hb_select_chunk": """
ctx, due = np.zeros(1 << 26, np.int32), np.full(1 << 26, 50.0)
model, chunk, ms = H.hb_latency_model(), C.c_int32(), C.c_double()
limit(1 << 28)
status = lib.hb_select_chunk(C.byref(model), C.byref(cfg), ctx.ctypes.data_as(C.POINTER(C.c_int32)),
                             due.ctypes.data_as(C.POINTER(C.c_double)), 1 << 26, 0.0, 0, 64, 32, 0.0,
                             C.byref(chunk), C.byref(ms))
""",
}


@pytest.mark.parametrize("name", CALLS)
def test_host_allocation_that_fails(name):
    code = COMMON % ROOT + CALLS[name] + "\nassert status == H.HB_ERR_OOM, status\nassert H.hb_last_error()\nprint('done')\n"
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "done", (r.returncode, r.stderr[-1500:])
