"""hs_set_window where the host has no memory left for the windows: an error code, and no exception into the caller's C (no GPU)."""
import os
import subprocess
import sys

import paper_2508_18588_amd as hs
from test_boundary_host import ROOT, lib  # noqa: F401  (the library fixture)

# a model of so many layers that its windows are an allocation of their own (16 MB), and no room for one
CHILD = r"""
import ctypes as C
import os
import resource
import paper_2508_18588_amd as hs
from test_boundary_host import _good

L = 1 << 22
desc, w, lim, _ = _good()
desc.n_layers = L
arr = (C.c_void_p * L)()
C.memset(arr, 0x10, C.sizeof(arr))
p = C.cast(arr, C.POINTER(C.c_void_p))
w = hs.hs_weights(0x1000, 0x1000, 0x1000, p, p, p, p, p, p, p, 0x1000)
ctx = hs.hs_create(desc, w, lim)
windows = (C.c_int32 * L)()
one = hs.lib().hs_set_window
with open("/proc/self/statm") as f:
    used = int(f.read().split()[0]) * os.sysconf("SC_PAGE_SIZE")
soft, hard = resource.getrlimit(resource.RLIMIT_AS)
resource.setrlimit(resource.RLIMIT_AS, (used + (2 << 20), hard))
first = one(ctx, windows, 3)
text = hs.lib().hs_last_error(ctx)
resource.setrlimit(resource.RLIMIT_AS, (soft, hard))
print(first, text.decode(), one(ctx, windows, 3), one(ctx, None, 0), flush=True)
"""


def test_no_memory_for_the_windows(lib):  # noqa: F811
    # (large allocations are mappings of their own, not what an earlier one has left in the heap)
    env = dict(os.environ, PYTHONPATH=f"{ROOT}:{ROOT}/tests", MALLOC_MMAP_THRESHOLD_=str(1 << 20))
    p = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                       text=True, timeout=120)
    assert p.returncode == 0, (p.returncode, p.stdout[-1000:])
    got = p.stdout.strip().splitlines()[-1]
    assert got.startswith(f"{hs.HS_ERR_CAPACITY} hs_set_window") and got.endswith(f" {hs.HS_OK} {hs.HS_OK}"), got
