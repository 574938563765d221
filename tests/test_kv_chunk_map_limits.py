"""pp_chunk_map at the largest counts: a status, never an exception through the C entry."""
import subprocess
import sys

import pytest

from paper_2608_01655_gb300 import build as ppbuild

# in a process of its own with 3 GB of address space beside what it has: an abort would end it
CODE = """
import ctypes, resource, sys
import numpy as np
from paper_2608_01655_gb300 import binding as pp
pages = int(open("/proc/self/statm").read().split()[0])
limit = pages * resource.getpagesize() + (3 << 30)
resource.setrlimit(resource.RLIMIT_AS, (limit, limit))
n = int(sys.argv[1])
a = lambda x, t: np.array([x], t).ctypes.data_as(ctypes.c_void_p)
out, used = np.zeros(4, np.int32), ctypes.c_int32(0)
print(pp._lib.pp_chunk_map(n, a(int(sys.argv[2]), np.int32), a(int(sys.argv[3]), np.int32), a(1, np.uint8), 1,
                           out.ctypes.data_as(ctypes.c_void_p), ctypes.byref(used)))
"""


@pytest.mark.parametrize("n,parent,weight,status", [
    ((1 << 31) - 1, -2, 1, 2), ((1 << 31) - 1, 0, 1, 2), ((1 << 31) - 1, -1, 0, 1), (1 << 30, 0, 1, 2), (1, -1, 1, 0)])
def test_chunk_map_checks_the_tree_before_it_allocates(n, parent, weight, status):
    """The first node is wrong, so the arrays' one element is all that is read."""
    ppbuild.build()
    r = subprocess.run([sys.executable, "-c", CODE, str(n), str(parent), str(weight)], capture_output=True, text=True,
                       cwd=ppbuild.ROOT)
    assert r.returncode == 0, r.stderr[-500:]
    assert int(r.stdout) == status
