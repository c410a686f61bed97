"""The list of an optimizer's step is looked through for params that stand in it twice without memory of its own, however long it is."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# A handle made by hand (a device's number and SMs, and its error word, which is not reached): every list has a param twice and is refused
# before anything asks for a device.
CHILD = """
import ctypes as C, resource, sys
import numpy as np
sys.path.insert(0, sys.argv[1])
from paper_2505_03983_b200 import operators as o
lib = o._library()
handle = (C.c_int64 * 2)(148 << 32, 0)
step = (C.c_int64 * 2)()
kind = np.dtype([("n", "i8"), ("types", "i8"), ("param", "u8"), ("grad", "u8"), ("master", "u8"), ("m", "u8"), ("v", "u8"), ("scales", "u8")])
assert kind.itemsize == C.sizeof(o._AdamwTensor)
big = 400000
t = np.zeros(big, kind)
t["n"], t["grad"], t["m"], t["v"] = 1, 64, 64, 64
places = 1024 + 512 * np.arange(big, dtype=np.uint64)
t["param"] = places

def call(count):
    a = o._Adamw(count=count, bits=32, tensors=C.cast(t.ctypes.data, C.POINTER(o._AdamwTensor)), lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=C.addressof(step))
    with open("/proc/self/statm") as f:
        size = int(f.read().split()[0]) * resource.getpagesize()
    resource.setrlimit(resource.RLIMIT_AS, (size + (1 << 18), resource.RLIM_INFINITY))
    status = lib.asd_adamw(C.addressof(handle), C.byref(a), None)
    resource.setrlimit(resource.RLIMIT_AS, (resource.RLIM_INFINITY,) * 2)
    return status, lib.asd_ops_last_error()

for count, pairs in ((2, [(0, 1)]), (300, [(0, 299), (150, 151)]), (2048, [(0, 2047)]), (2049, [(0, 2048), (2047, 2048)]), (4500, [(0, 4499), (2047, 2048), (2050, 4096), (4498, 4499)]),
                     (big, [(0, big - 1), (big - 2, big - 1), (1000, 300000)])):
    for i, j in pairs:
        own = t["param"][j]
        t["param"][j] = t["param"][i]
        status, message = call(count)
        assert status == 1 and message == b"tensor %d: its param stands in the list twice" % j, (count, i, j, status, message)
        if count > 4:  # without elements nothing is changed twice: what the list is then refused for is another pair
            t["n"][i], x, y = 0, *[k for k in range(5) if k not in (i, j)][:2]
            t["param"][y] = t["param"][x]
            assert call(count) == (1, b"tensor %d: its param stands in the list twice" % y), (count, i, j)
        t["n"] = 1
        t["param"] = places
print("done")
"""


@pytest.mark.skipif(not sys.platform.startswith("linux"), reason="limits the process's memory as Linux does")
def test_a_long_list_needs_no_memory():
    from paper_2505_03983_b200 import build
    build.build()
    r = subprocess.run([sys.executable, "-c", CHILD, ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "done" in r.stdout, r.stdout + r.stderr
