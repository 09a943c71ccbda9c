"""Planning where the host has no memory left: an error, not the end of the process."""
import subprocess
import sys

import pytest

CHILD = """
import ctypes, resource, sys
import numpy as np
from paper_2412_07017_b200 import binding as B
from paper_2412_07017_b200.workload import Shape

lib, kind = B.load(), sys.argv[1]
rows = 3_000_000                                   # of one new token each: with 64 kv heads 192 M units
q_indptr = np.arange(rows + 1, dtype=np.int32)
ctx, page_indptr, pages = np.zeros(rows, np.int32), np.arange(rows + 1, dtype=np.int32), np.zeros(rows, np.int32)
groups = [(0, 2, 0)] if kind == "prefix" else None
make = B._planner(Shape(64, 64, 64, 16), 8, q_indptr, ctx, page_indptr, pages, 0.0, groups, (4, 1, 1) if kind == "sparse" else None, num_sms=148)
ws = np.zeros(1 << 20, np.int64)
out = ctypes.c_void_p()
used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (used + (512 << 20), resource.RLIM_INFINITY))
print("status", make(ws.ctypes.data, ws.nbytes, None, 0, None, ctypes.byref(out))[0], flush=True)
"""


@pytest.mark.parametrize("kind", ["plain", "prefix", "sparse"])
def test_no_memory_is_an_error(kind):
    p = subprocess.run([sys.executable, "-c", CHILD, kind], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout.split() == ["status", "-9"], (p.returncode, p.stdout, p.stderr[-300:])
