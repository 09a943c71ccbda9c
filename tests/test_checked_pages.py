"""The checked build of the library (-DASYNCLM_DEBUG) and the calls of selected pages: a page id beyond the pool sets the plan's status word and is not used.
The bad ids are written into plans' device copies in a child process that has loaded the checked build only."""
import json
import os
import subprocess
import sys

import pytest

from paper_2412_07017_b200 import build as lib_build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.gpu
def test_bad_page_ids_of_bounds_and_selections():
    lib = lib_build.DEBUG_LIB
    inputs = lib_build.sources() + [os.path.join(lib_build.CSRC, f) for f in os.listdir(lib_build.CSRC) if f.endswith((".cuh", ".h"))]
    if not os.path.exists(lib) or any(os.path.getmtime(f) > os.path.getmtime(lib) for f in inputs):
        lib = lib_build.build(debug=True)
    proc = subprocess.run([sys.executable, os.path.join(HERE, "checked_pages_child.py")], env=dict(os.environ, ASYNCLM_LIBRARY=lib), capture_output=True, text=True,
                          timeout=600)
    assert proc.returncode == 0, proc.stdout + proc.stderr
    res = json.loads(proc.stdout.strip().splitlines()[-1])
    assert res == {f"{what} {kv8}": code for kv8 in (False, True) for what, code in (("bounds", 46), ("select", 47), ("equal", 47))}, res
