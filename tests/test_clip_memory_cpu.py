"""picospec_clip_grad where the host has no memory for the list that many tensors are checked with: an error of its own, not that of a bad argument."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import ctypes as C, resource, sys
from paper_2603_19133_amd import binding as B
n = 1 << 23
grads, numel, dtypes = (C.c_void_p * n)(), (C.c_int64 * n)(), (C.c_int32 * n)()        # (tensors without elements)
call = lambda: B.lib.picospec_clip_grad(n, grads, None, numel, dtypes, 1.0, 0x1000, None, 0, None)
assert call() == B.EWORKSPACE
now = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (now + (64 << 20),) * 2)                        # (the list has 256 MB)
sys.exit(0 if call() == B.EUNSUPPORTED else 1)
"""


def test_no_memory_for_the_list():
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
